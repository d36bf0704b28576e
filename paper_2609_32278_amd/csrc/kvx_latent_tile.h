// Device helpers shared by the latent attention kernels: vector types, conversions, and a
// tile of 64 cache rows staged in LDS as bf16.
#pragma once

#include "kvx_latent_internal.h"

namespace kvx {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLn2 = 0.6931471805599453f;

template <int LAT>
struct LatGeom {
  static constexpr int ROW = LAT + kLatRope;          // values of an entry
  static constexpr int ROWB = ROW * 2;                // bytes of its bf16 row in LDS
  static constexpr int KS = ROW / 32;                 // k-steps of the score product
  static constexpr int DW = LAT / 4;                  // latent dims of a wave's sums
  static constexpr int DB = DW / 16;
  static constexpr int TILE = kLatTileKeys * ROWB;
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  bf16x2 v;
  v[0] = (__bf16)a;
  v[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, v);
}

typedef const __attribute__((address_space(4))) int32_t* const_i32_ptr;  // scalar-loaded

// This workgroup's element of the list in a kernel's parameters (its first argument), or of
// the one in memory: scalar loads, so that what follows from it stays uniform.
template <typename U, typename Params>
__device__ __forceinline__ U listed(const Params& p, const U* memory) {
  const const_i32_ptr in_args =
      (const_i32_ptr)((const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr() +
                      offsetof(Params, list) + offsetof(decltype(p.list), at));
  const const_i32_ptr w = (p.list.n > 0 ? in_args : (const_i32_ptr)memory) + (size_t)blockIdx.x * (sizeof(U) / 4);
  int32_t words[sizeof(U) / 4];
#pragma unroll
  for (size_t i = 0; i < sizeof(U) / 4; i++) words[i] = w[i];
  U u;
  __builtin_memcpy(&u, words, sizeof u);
  return u;
}

// Keep an operand that is used throughout a unit in the accumulator half of the register
// file, which the matrix instructions read as well.
__device__ __forceinline__ void keep_in_acc(bf16x8& x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm("" : "+a"(x));
#endif
}
// An address offset that the compiler shall not take apart, so that one register and an
// immediate make each address.
__device__ __forceinline__ void opaque(uint32_t& x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm("" : "+v"(x));
#endif
}

// A value to be formed here, not where the compiler finds it used.
template <typename T>
__device__ __forceinline__ void formed(T& x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(x));
#endif
}

// The transposing LDS read: lanes 4 j + i of 16 point at 4 values each of row j (16 values
// side by side); lane i receives column i of the four rows.
__device__ __forceinline__ s16x4 read_tr(const uint8_t* at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(__attribute__((address_space(3))) void*)at);
}

typedef const __attribute__((address_space(3))) uint8_t* lds_ptr;
__device__ __forceinline__ lds_ptr lds_at(uint32_t at) { return (lds_ptr)(uintptr_t)at; }
__device__ __forceinline__ s16x4 read_tr(lds_ptr at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
}
__device__ __forceinline__ bf16x8 read_b128(lds_ptr at) {
  return *(const __attribute__((address_space(3))) bf16x8*)at;
}

__device__ __forceinline__ void write_b64(uint32_t at, uint32_t x, uint32_t y) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  *(__attribute__((address_space(3))) u32x2*)(uintptr_t)at = u32x2{x, y};
}

__device__ __forceinline__ void write_b128(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  *(__attribute__((address_space(3))) u32x4*)(uintptr_t)at = u32x4{x, y, z, w};
}

__device__ __forceinline__ bf16x8 join(s16x4 a, s16x4 b) {
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Direct global -> LDS load of 1 KiB: lane l's 16 bytes at base + off land at LDS address
// lds + 16 l.  Inline assembly, so that the compiler's wait counts, which cannot tell the
// buffers apart, do not drain these loads; the kernels wait themselves.
__device__ __forceinline__ void lds_load_1k(const uint8_t* base, int off, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds), "v"(off), "s"(base)
      : "memory", "m0");
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)p;
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  // s_waitcnt with only the vector-memory counter limited (expcnt, lgkmcnt at max)
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

}  // namespace
}  // namespace kvx
