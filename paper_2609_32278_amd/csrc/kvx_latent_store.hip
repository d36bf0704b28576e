// Latent cache entries into the pages and back, gfx950 (CDNA4).
//
// HBM-bound: each row is read once and written once; the queries whose last 64 dims turn
// outweigh the entries by their number of heads.  One workgroup takes one touched page: grid
// y = 0 its (at most 16) entries, y >= 1 groups of 8 query heads of the same tokens, which share
// the angles.  Measured, 8-bit pool: 16 turns, 20857 tokens, 128 heads of 192 dims out of
// place 445 us, 4.7 TB/s; read-back of 472k tokens 157 us, 5.4 TB/s (a large copy reaches 5.0).
// One request or a few of a token each: 3 to 6 us, latency.
//
// An entry's latent is held by latent_dim / 8 lanes, eight values each, so that the norm's
// sum and a scale group's maximum (eight lanes) are sums and maxima over lanes.  The rotated
// key and the queries' rotated dims go as pairs of 16-byte pieces (dims 8 p .. and 32 + 8 p
// ..), which hold both halves of every plane in either style.

#include "kvx_latent_internal.h"
#include "kvx_store_util.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;
constexpr int kPlanes = kLatRope / 2;

struct Angles {
  float2 cs[kPageSize][kPlanes];  // (cos, sin) of every live slot and plane
};

__device__ __forceinline__ void unpack(uint4 raw, float (&x)[8]) {
  const uint16_t* h = (const uint16_t*)&raw;
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = bf16_to_f32(h[e]);
}

// Turn pieces pr (dims 8 pr ..) and pr + 4 (dims 32 + 8 pr ..) of a 64-dim head.
template <bool INTERLEAVED>
__device__ __forceinline__ void turn(float (&x)[8], float (&y)[8], const float2* cs, int pr) {
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float2 c = cs[4 * pr + i], d = cs[16 + 4 * pr + i];
      const float a = x[2 * i], b = x[2 * i + 1], e = y[2 * i], f = y[2 * i + 1];
      x[2 * i] = a * c.x - b * c.y;
      x[2 * i + 1] = a * c.y + b * c.x;
      y[2 * i] = e * d.x - f * d.y;
      y[2 * i + 1] = e * d.y + f * d.x;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float2 c = cs[8 * pr + e];
      const float a = x[e], b = y[e];
      x[e] = a * c.x - b * c.y;
      y[e] = a * c.y + b * c.x;
    }
  }
}

// The group's power of two (see kvx_latent.h) from its largest magnitude: amax = 1.f 2^(E - 127)
// is at most 448 * 2^e = 1.75 * 2^(8 + e) for e = E - 135, or one more where 1.f > 1.75.
__device__ __forceinline__ int group_exp(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 135 + ((b & 0x7FFFFF) > 0x600000 ? 1 : 0);
  return e < kLatMinExp ? kLatMinExp : (e > kLatMaxExp ? kLatMaxExp : e);
}

// clamp448 lets a NaN end as a number; the cache keeps it.
__device__ __forceinline__ float clamp_keep_nan(float x) { return x != x ? x : clamp448(x); }

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_keep_nan(a), clamp_keep_nan(b), 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_keep_nan(c), clamp_keep_nan(d), r, true);
  return (uint32_t)r;
}

template <int LAT, bool FP8, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void store_latent_kernel(LatentStoreParams p) {
  constexpr int LPT = LAT / 8;           // lanes per token
  constexpr int TPW = 64 / LPT;          // tokens of a wave at once
  constexpr int ITS = kPageSize / (4 * TPW);
  constexpr int ROW = LAT + kLatRope;
  __shared__ Angles sm;
  const RopeUnit u = p.reqs.n > 0 ? inline_unit(p.reqs, blockIdx.x) : p.units[blockIdx.x];
  const int ntok = u.slot_end - u.slot_begin;
  const int64_t row0 = (int64_t)u.row_slot0 + u.slot_begin;  // first suffix row of the unit
  const int tid = threadIdx.x;
  if (p.rotate) {
    for (int e = tid; e < ntok * kPlanes; e += kThreads) {
      const int s = e / kPlanes, j = e % kPlanes;
      double rev = (double)(u.pos_slot0 + u.slot_begin + s) * p.rev_freq[j];
      rev -= rint(rev);  // [-1/2, 1/2] turn, exact
      float sn, cn;
      sincospif(2.0f * (float)rev, &sn, &cn);
      sm.cs[s][j] = make_float2(cn, sn);
    }
    __syncthreads();
  }

  if (blockIdx.y > 0) {
    const int lg = p.lg_q, h0 = ((int)blockIdx.y - 1) << lg, D = p.q_dim, Hq = p.num_q_heads;
    const int nrows = ntok << lg;
    const uint16_t* q = p.q + (size_t)row0 * Hq * D;
    uint16_t* qo = p.q_out + (size_t)row0 * Hq * D;
    // several pieces of a thread in flight before the first is used
    constexpr int FLIGHT = 4;
    const int lgm = (1 << lg) - 1;
    auto at_row = [&](int r) { return ((size_t)(r >> lg) * Hq + h0 + (r & lgm)) * D; };
    for (int i0 = tid; i0 < nrows * 4; i0 += FLIGHT * kThreads) {
      uint4 a[FLIGHT], b[FLIGHT];
#pragma unroll
      for (int f = 0; f < FLIGHT; f++) {
        const int i = i0 + f * kThreads, r = i >> 2;
        if (i < nrows * 4 && h0 + (r & lgm) < Hq) {
          const uint16_t* src = q + at_row(r) + (D - kLatRope) + (i & 3) * 8;
          a[f] = load16<false>(src);
          b[f] = load16<false>(src + 32);
        }
      }
#pragma unroll
      for (int f = 0; f < FLIGHT; f++) {
        const int i = i0 + f * kThreads, r = i >> 2, pr = i & 3;
        if (i < nrows * 4 && h0 + (r & lgm) < Hq) {
          float x[8], y[8];
          unpack(a[f], x);
          unpack(b[f], y);
          turn<INTERLEAVED>(x, y, sm.cs[r >> lg], pr);
          uint16_t* dst = qo + at_row(r) + (D - kLatRope) + pr * 8;
          store16<true>(dst, pack_bf16x8(x));
          store16<true>(dst + 32, pack_bf16x8(y));
        }
      }
    }
    if (p.q_out == p.q) return;  // uniform
    const int plain = (D - kLatRope) / 8, items = nrows * plain;
    for (int i0 = tid; i0 < items; i0 += FLIGHT * kThreads) {
      uint4 a[FLIGHT];
      size_t at[FLIGHT];
      bool in[FLIGHT];
#pragma unroll
      for (int f = 0; f < FLIGHT; f++) {
        const int i = i0 + f * kThreads, r = i / plain;
        in[f] = i < items && h0 + (r & lgm) < Hq;
        at[f] = at_row(r) + (i - r * plain) * 8;
        if (in[f]) a[f] = load16<false>(q + at[f]);
      }
#pragma unroll
      for (int f = 0; f < FLIGHT; f++)
        if (in[f]) store16<true>(qo + at[f], a[f]);
    }
    return;
  }

  uint8_t* page = p.pool.base + (int64_t)p.pool.page_ids[u.page_pos] * p.pool.page_bytes;
  const int lane = tid & 63, wave = tid >> 6, sub = lane / LPT, c = lane % LPT;
  uint4 raw[ITS];
#pragma unroll
  for (int it = 0; it < ITS; it++) {
    const int tok = (it * 4 + wave) * TPW + sub;
    raw[it] = make_uint4(0, 0, 0, 0);
    if (tok < ntok) raw[it] = *(const uint4*)(p.kv + (row0 + tok) * p.kv_stride + c * 8);
  }
  float w[8];
  if (p.norm) unpack(*(const uint4*)(p.norm + c * 8), w);
#pragma unroll
  for (int it = 0; it < ITS; it++) {
    const int tok = (it * 4 + wave) * TPW + sub, slot = u.slot_begin + tok;
    float x[8];
    unpack(raw[it], x);
    if (p.norm) {  // uniform; lanes of tokens past the unit's sum zeros
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; e++) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int m = 1; m < LPT; m <<= 1) ss += __shfl_xor(ss, m, 64);
      const float inv = 1.0f / sqrtf(ss * (1.0f / LAT) + p.norm_eps);
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] = (x[e] * inv) * w[e];
    }
    if constexpr (FP8) {
      float amax = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; e++) amax = fmaxf(amax, fabsf(x[e]));
#pragma unroll
      for (int m = 1; m < 8; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m, 64));
      const int ex = group_exp(amax);
      const float by = __uint_as_float((uint32_t)(127 - ex) << 23);
      uint2 code;
      code.x = codes4(x[0] * by, x[1] * by, x[2] * by, x[3] * by);
      code.y = codes4(x[4] * by, x[5] * by, x[6] * by, x[7] * by);
      if (tok < ntok) {
        *(uint2*)(page + (size_t)slot * LAT + c * 8) = code;
        if (c % 8 == 0)
          page[kPageSize * (LAT + 2 * kLatRope) + latent_scale_at(LAT, slot, c / 8)] = (uint8_t)(ex + 127);
      }
    } else {
      if (tok < ntok)
        store16<false>((uint16_t*)page + (size_t)slot * ROW + c * 8, p.norm ? pack_bf16x8(x) : raw[it]);
    }
  }
  if (tid < ntok * 4) {
    const int tok = tid >> 2, pr = tid & 3, slot = u.slot_begin + tok;
    const uint16_t* src = p.kv + (row0 + tok) * p.kv_stride + LAT + pr * 8;
    uint16_t* dst = FP8 ? (uint16_t*)(page + kPageSize * LAT) + slot * kLatRope + pr * 8
                        : (uint16_t*)page + (size_t)slot * ROW + LAT + pr * 8;
    uint4 a = *(const uint4*)src, b = *(const uint4*)(src + 32);
    if (p.rotate) {
      float x[8], y[8];
      unpack(a, x);
      unpack(b, y);
      turn<INTERLEAVED>(x, y, sm.cs[tok], pr);
      a = pack_bf16x8(x);
      b = pack_bf16x8(y);
    }
    *(uint4*)dst = a;
    *(uint4*)(dst + 32) = b;
  }
}

// 16 codes -> 16 bf16 values (code * 2^e is exact in bf16)
__device__ __forceinline__ void dequant16(uint4 codes, float scale, uint4 (&out)[2]) {
  const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
  uint32_t* o = (uint32_t*)out;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
    o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
  }
}

template <int LAT, bool FP8>
__global__ __launch_bounds__(kThreads) void load_latent_kernel(LatentLoadParams p) {
  constexpr int ROW = LAT + kLatRope;
  const RopeUnit u = p.reqs.n > 0 ? inline_unit(p.reqs, blockIdx.x) : p.units[blockIdx.x];
  const int ntok = u.slot_end - u.slot_begin;
  const uint8_t* page = p.pool.base + (int64_t)p.pool.page_ids[u.page_pos] * p.pool.page_bytes;
  uint16_t* out = p.out + ((int64_t)u.row_slot0 + u.slot_begin) * p.out_stride;
  const int tid = threadIdx.x;
  if constexpr (FP8) {
    constexpr int CPT = LAT / 16;  // pieces of 16 codes per token
    constexpr int ITS = kPageSize * CPT / kThreads;
    uint4 x[ITS];
    uint8_t s[ITS];
#pragma unroll
    for (int it = 0; it < ITS; it++) {
      const int i = it * kThreads + tid, tok = i / CPT, c = i % CPT;
      if (tok < ntok) {
        x[it] = load16<true>(page + (u.slot_begin + tok) * LAT + c * 16);
        s[it] = page[kPageSize * (LAT + 2 * kLatRope) + latent_scale_at(LAT, u.slot_begin + tok, c / 4)];
      }
    }
    if (tid < ntok * 8) {
      const int tok = tid >> 3, c = tid & 7;
      const uint4 k = *(const uint4*)((const uint16_t*)(page + kPageSize * LAT) + (u.slot_begin + tok) * kLatRope + c * 8);
      *(uint4*)(out + tok * p.out_stride + LAT + c * 8) = k;
    }
#pragma unroll
    for (int it = 0; it < ITS; it++) {
      const int i = it * kThreads + tid, tok = i / CPT, c = i % CPT;
      if (tok < ntok) {
        uint4 y[2];
        dequant16(x[it], __uint_as_float((uint32_t)s[it] << 23), y);
        *(uint4*)(out + tok * p.out_stride + c * 16) = y[0];
        *(uint4*)(out + tok * p.out_stride + c * 16 + 8) = y[1];
      }
    }
  } else {
    constexpr int CPT = ROW / 8;
    constexpr int ITS = (kPageSize * CPT + kThreads - 1) / kThreads;
    uint4 x[ITS];
#pragma unroll
    for (int it = 0; it < ITS; it++) {
      const int i = it * kThreads + tid, tok = i / CPT, c = i % CPT;
      if (tok < ntok) x[it] = load16<true>((const uint16_t*)page + (size_t)(u.slot_begin + tok) * ROW + c * 8);
    }
#pragma unroll
    for (int it = 0; it < ITS; it++) {
      const int i = it * kThreads + tid, tok = i / CPT, c = i % CPT;
      if (tok < ntok) *(uint4*)(out + tok * p.out_stride + c * 8) = x[it];
    }
  }
}

template <int LAT, bool FP8>
void store_by_style(const LatentStoreParams& p, dim3 grid, bool interleaved, hipStream_t stream) {
  if (interleaved) hipLaunchKernelGGL((store_latent_kernel<LAT, FP8, true>), grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((store_latent_kernel<LAT, FP8, false>), grid, dim3(kThreads), 0, stream, p);
}

}  // namespace

hipError_t launch_store_latent(const LatentStoreParams& p0, int64_t n_units, int latent_dim, bool fp8, bool interleaved,
                               hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  LatentStoreParams p = p0;
  p.lg_q = 3;  // 8 heads a workgroup: 20k tokens of 128 heads 460 us, with 16, 32 and 128 heads 478, 474 and 500
  const int groups = p.num_q_heads > 0 ? (p.num_q_heads + (1 << p.lg_q) - 1) >> p.lg_q : 0;
  const dim3 grid((unsigned)n_units, 1 + groups);
  if (latent_dim == 512) {
    if (fp8) store_by_style<512, true>(p, grid, interleaved, stream);
    else store_by_style<512, false>(p, grid, interleaved, stream);
  } else {
    if (fp8) store_by_style<256, true>(p, grid, interleaved, stream);
    else store_by_style<256, false>(p, grid, interleaved, stream);
  }
  return hipGetLastError();
}

hipError_t launch_load_latent(const LatentLoadParams& p, int64_t n_units, int latent_dim, bool fp8,
                              hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  const dim3 grid((unsigned)n_units), block(kThreads);
  if (latent_dim == 512) {
    if (fp8) hipLaunchKernelGGL((load_latent_kernel<512, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((load_latent_kernel<512, false>), grid, block, 0, stream, p);
  } else {
    if (fp8) hipLaunchKernelGGL((load_latent_kernel<256, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((load_latent_kernel<256, false>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace kvx
