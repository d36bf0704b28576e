// Device helpers of the store kernels: 16-byte accesses, bf16 and e4m3 conversions, and the
// unit of a workgroup whose batch travels in the kernel arguments.
#pragma once

#include "kvx_internal.h"

namespace kvx {
namespace {

// 16-byte accesses; NT: non-temporal, for data that no cache need keep.
template <bool NT>
__device__ __forceinline__ uint4 load16(const void* p) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  if constexpr (NT) return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4*)p));
  else return *(const uint4*)p;
}
template <bool NT>
__device__ __forceinline__ void store16(void* p, uint4 x) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), (u32x4*)p);
  else *(uint4*)p = x;
}

__device__ __forceinline__ float bf16_to_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

__device__ __forceinline__ float clamp448(float x) { return fminf(fmaxf(x, -448.0f), 448.0f); }

// 4 floats -> 4 e4m3 codes (byte i = value i)
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(a), clamp448(b), 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(c), clamp448(d), r, true);
  return (uint32_t)r;
}

__device__ __forceinline__ uint4 pack_bf16x8(const float (&y)[8]) {
  uint4 r;
  uint32_t* w = (uint32_t*)&r;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const __bf16 lo = (__bf16)y[2 * i], hi = (__bf16)y[2 * i + 1];
    w[i] = (uint32_t)__builtin_bit_cast(uint16_t, lo) | ((uint32_t)__builtin_bit_cast(uint16_t, hi) << 16);
  }
  return r;
}

// The unit of workgroup b of a small batch (see StoreReqs); uniform.
__device__ __forceinline__ RopeUnit inline_unit(const StoreReqs& rq, int b) {
  int lo = 0, hi = rq.n;  // request r with first[r] <= b < first[r + 1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (rq.first[mid] <= b) lo = mid;
    else hi = mid;
  }
  const int P = rq.prefix[lo], L = rq.end[lo];
  const int lp = P / kPageSize + (b - rq.first[lo]);
  RopeUnit u;
  u.pos_slot0 = lp * kPageSize;
  u.row_slot0 = rq.qo[lo] + u.pos_slot0 - P;
  u.page_pos = rq.page_base[lo] + lp;
  u.slot_begin = (P > u.pos_slot0 ? P : u.pos_slot0) - u.pos_slot0;
  u.slot_end = (L < u.pos_slot0 + kPageSize ? L : u.pos_slot0 + kPageSize) - u.pos_slot0;
  return u;
}

}  // namespace
}  // namespace kvx
