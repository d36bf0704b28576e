// Products with the per-head weights of latent attention, gfx950: queries into the latent
// space and sums out of it (absorbed form), cached rows to keys and values (expanded form).
#include "kvx_latent_tile.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;
constexpr int kSlice = 128;  // latent dims per workgroup of the query product

// q' = W_uk^T q, as (W_uk^T) q^T: W's rows run along the latent dims, so its operand is read
// transposed from LDS.  Workgroup: 64 tokens, one head, 128 latent dims.
template <int LAT, int D>
__global__ __launch_bounds__(kThreads) void latent_absorb_kernel(LatentProjParams p) {
  constexpr int IN = D + kLatRope, OUT = LAT + kLatRope;
  constexpr int WB = kSlice * 2 + 32;  // LDS row
  __shared__ __attribute__((aligned(16))) uint8_t wl[D * WB];
  const LatentRows rows = listed(p, p.rows);
  const int hd = blockIdx.y, s0 = blockIdx.z * kSlice;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
  const uint16_t* w = p.w + (size_t)hd * D * LAT + s0;
  for (int i = tid; i < D * (kSlice / 8); i += kThreads) {
    const int k = i / (kSlice / 8), c = i % (kSlice / 8);
    *(uint4*)(wl + k * WB + c * 16) = *(const uint4*)(w + (size_t)k * LAT + c * 8);
  }
  __syncthreads();
  f32x4 acc[4][2];
#pragma unroll
  for (int tb = 0; tb < 4; tb++) acc[tb][0] = acc[tb][1] = f32x4{};
  const uint16_t* q[4];
#pragma unroll
  for (int tb = 0; tb < 4; tb++) {
    const int t = tb * 16 + n;
    q[tb] = p.in + ((size_t)(rows.row0 + (t < rows.ntok ? t : 0)) * p.num_q_heads + hd) * IN;
  }
#pragma unroll
  for (int ks = 0; ks < D / 32; ks++) {
    bf16x8 a[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
      s16x4 h[2];
#pragma unroll
      for (int e = 0; e < 2; e++)
        h[e] = read_tr(wl + (ks * 32 + 8 * g + 4 * e + n / 4) * WB + (wave * 32 + b * 16) * 2 + (n % 4) * 8);
      a[b] = join(h[0], h[1]);
    }
#pragma unroll
    for (int tb = 0; tb < 4; tb++) {
      const bf16x8 x = *(const bf16x8*)(q[tb] + ks * 32 + 8 * g);
#pragma unroll
      for (int b = 0; b < 2; b++) acc[tb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[b], x, acc[tb][b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int tb = 0; tb < 4; tb++) {
    const int t = tb * 16 + n;
    if (t >= rows.ntok) continue;
    uint16_t* dst = p.out + ((size_t)(rows.own0 + t) * p.num_q_heads + hd) * OUT;
#pragma unroll
    for (int b = 0; b < 2; b++) {
      uint2 y;
      y.x = pack_bf16(acc[tb][b][0], acc[tb][b][1]);
      y.y = pack_bf16(acc[tb][b][2], acc[tb][b][3]);
      *(uint2*)(dst + s0 + wave * 32 + b * 16 + 4 * g) = y;
    }
    if (blockIdx.z == 0) {  // the rotated dims follow: 8 chunks, two of them per (wave, g) of waves 0
      if (wave == 0) {
#pragma unroll
        for (int c = 0; c < 2; c++) *(uint4*)(dst + LAT + (2 * g + c) * 8) = *(const uint4*)(q[tb] + D + (2 * g + c) * 8);
      }
    }
  }
}

// o = W_uv (sum), as W_uv o^T; both operands run along the latent dims.  Workgroup: 64
// tokens, one head.
template <int LAT, int D>
__global__ __launch_bounds__(kThreads) void latent_output_kernel(LatentProjParams p) {
  constexpr int NB = D / 64;  // 16-row blocks of W per wave
  const LatentRows rows = listed(p, p.rows);
  const int hd = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
  const uint16_t* w = p.w + ((size_t)hd * D + wave * (D / 4) + n) * LAT + 8 * g;
  const uint16_t* x[4];
  f32x4 acc[4][NB];
#pragma unroll
  for (int tb = 0; tb < 4; tb++) {
    const int t = tb * 16 + n;
    x[tb] = p.in + ((size_t)(rows.own0 + (t < rows.ntok ? t : 0)) * p.num_q_heads + hd) * LAT + 8 * g;
#pragma unroll
    for (int b = 0; b < NB; b++) acc[tb][b] = f32x4{};
  }
#pragma unroll 4
  for (int ks = 0; ks < LAT / 32; ks++) {
    bf16x8 a[NB];
#pragma unroll
    for (int b = 0; b < NB; b++) a[b] = *(const bf16x8*)(w + (size_t)b * 16 * LAT + ks * 32);
#pragma unroll
    for (int tb = 0; tb < 4; tb++) {
      const bf16x8 y = *(const bf16x8*)(x[tb] + ks * 32);
#pragma unroll
      for (int b = 0; b < NB; b++) acc[tb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[b], y, acc[tb][b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int tb = 0; tb < 4; tb++) {
    const int t = tb * 16 + n;
    if (t >= rows.ntok) continue;
    uint16_t* dst = p.out + ((size_t)(rows.row0 + t) * p.num_q_heads + hd) * D + wave * (D / 4) + 4 * g;
    if (p.lse_out != nullptr && wave == 0 && g == 0)
      p.lse_out[(size_t)(rows.row0 + t) * p.num_q_heads + hd] = p.lse_in[(size_t)(rows.own0 + t) * p.num_q_heads + hd];
#pragma unroll
    for (int b = 0; b < NB; b++) {
      uint2 y;
      y.x = pack_bf16(acc[tb][b][0], acc[tb][b][1]);
      y.y = pack_bf16(acc[tb][b][2], acc[tb][b][3]);
      *(uint2*)(dst + b * 16) = y;
    }
  }
}

// Keys and values of cached tokens: (tokens x latent) times (latent x 2 head_dim) per head.
// Workgroup = 8 waves: 256 tokens against the columns of W_uk and W_uv of one head after the
// other, 64 latent dims a step, both operands double-buffered in LDS so that the loads of a
// step (those of the next head's first step too) arrive under the products of the one before.
// Waves 2 i and 2 i + 1 take 64 tokens, one W_uk, the other W_uv.
//
// LDS layout of a step: groups of 8 rows of 64 values, [8 rows][128 bytes] each, filled by one
// wave-wide direct load; 16-byte chunk c of row r is stored at c ^ x(r), x from row bits 1 to 3
// for tokens and 1, 2, 4 for weights: the rows that 16 lanes read together differ in those.
constexpr int kExpThreads = 512;
constexpr int kExpTok = kLatExpandTok;
__device__ __forceinline__ int wswz(int r) { return ((r >> 1) & 3) | ((r >> 2) & 4); }

template <int LAT, int D, bool FP8>
__global__ __launch_bounds__(kExpThreads, 1) void latent_expand_kernel(LatentExpandParams p) {
  constexpr int MB = D / 32;               // 32-row blocks of a wave's weights
  constexpr int STEPS = LAT / 64;
  constexpr int A_BYTES = kExpTok * 128, W_BYTES = 2 * D * 128, STAGE = A_BYTES + W_BYTES;
  constexpr int WG = 2 * D / 64;           // groups of 8 weight rows per wave
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  const LatentExpandUnit u = listed(p, p.units);
  const int head0 = blockIdx.y * p.heads_per, heads = p.heads - head0 < p.heads_per ? p.heads - head0 : p.heads_per;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int32_t* ids = p.pool.page_ids + u.page_base;
  const int last = u.key_end - 1;

  if (p.rx != nullptr && blockIdx.y == 0) {
    for (int i = tid; i < u.nrows * 8; i += kExpThreads) {
      const int r = i / 8, c = i % 8, key = u.key0 + r < last ? u.key0 + r : last;
      const uint8_t* page = p.pool.base + (int64_t)ids[key / kPageSize] * p.pool.page_bytes;
      const uint8_t* src = FP8 ? page + kPageSize * LAT + (key % kPageSize) * (2 * kLatRope)
                               : page + (key % kPageSize) * (2 * (LAT + kLatRope)) + 2 * LAT;
      *(uint4*)(p.rx + (size_t)(u.x_row + r) * kLatRope + c * 8) = *(const uint4*)(src + c * 16);
    }
  }

  // tokens: wave w stages rows 32 w .. 32 w + 31
  const uint8_t* a_src[4];
  uint4 codes[2];
  uint8_t sc[2];
  if constexpr (FP8) {
#pragma unroll
    for (int i = 0; i < 2; i++) {  // 16 codes a lane: row 32 wave + 16 i + lane / 4
      const int r = u.key0 + wave * 32 + i * 16 + lane / 4, key = r < last ? r : last;
      a_src[i] = p.pool.base + (int64_t)ids[key / kPageSize] * p.pool.page_bytes + (key % kPageSize) * LAT + (lane % 4) * 16;
      const int slot = key % kPageSize;
      a_src[2 + i] = a_src[i] - (slot * LAT + (lane % 4) * 16) + kPageSize * (LAT + 2 * kLatRope) + latent_scale_at(LAT, slot, 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = u.key0 + wave * 32 + i * 8 + lane / 8, key = r < last ? r : last;
      a_src[i] = p.pool.base + (int64_t)ids[key / kPageSize] * p.pool.page_bytes +
                 (key % kPageSize) * (2 * (LAT + kLatRope)) + (((lane & 7) ^ swz(i * 8 + lane / 8)) << 4);
    }
  }
  const int w_off = (lane >> 3) * (LAT * 2) + (((lane & 7) ^ ((lane >> 4) & 3)) << 4);
  const uint32_t base = lds_address(lds);
  // step i of the workgroup: head head0 + i / STEPS, latent dims 64 (i % STEPS) ..
  auto issue = [&](int i) {
    const int hd = head0 + i / STEPS, k0 = i % STEPS * 64;
    const uint32_t at = base + (i & 1) * STAGE;
    if constexpr (FP8) {
#pragma unroll
      for (int j = 0; j < 2; j++) {
        codes[j] = *(const uint4*)(a_src[j] + k0);
        sc[j] = a_src[2 + j][(k0 / 64 & 1) * (LAT / 64) + k0 / 128];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) lds_load_1k(a_src[j] + k0 * 2, at + (wave * 4 + j) * 1024);
    }
#pragma unroll
    for (int j = 0; j < WG; j++) {
      const int gr = wave * WG + j;  // rows 8 gr ..: W_uk's, then W_uv's
      const uint16_t* w = gr * 8 < D ? p.w_uk + ((size_t)hd * D + gr * 8) * LAT : p.w_uv + ((size_t)hd * D + gr * 8 - D) * LAT;
      lds_load_1k((const uint8_t*)(w + k0), w_off ^ ((gr >> 1) & 1) << 6, at + A_BYTES + gr * 1024);
    }
  };
  auto finish = [&](int i) {
    if constexpr (FP8) {
      uint8_t* at = lds + (i & 1) * STAGE;
#pragma unroll
      for (int j = 0; j < 2; j++) {
        const int r = wave * 32 + j * 16 + lane / 4, c = (lane % 4) * 2;
        const float s = __uint_as_float((uint32_t)sc[j] << 23);
        const uint32_t w[4] = {codes[j].x, codes[j].y, codes[j].z, codes[j].w};
        uint32_t y[8];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          y[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], s, false));
          y[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], s, true));
        }
        *(uint4*)(at + r * 128 + ((c ^ swz(r)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
        *(uint4*)(at + r * 128 + (((c + 1) ^ swz(r)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
      }
    }
  };

  const int rows0 = (wave >> 1) * 64, is_v = wave & 1;
  // Weight row of MFMA row m: lane (n, h) of the result then holds 16 values side by side.
  const int mw = (n & 3) | ((n & 4) << 2) | ((n >> 1) & 12);
  uint32_t aat[4], wat[4];
#pragma unroll
  for (int ks = 0; ks < 4; ks++) {
    aat[ks] = base + (rows0 + n) * 128 + (((2 * ks + h) ^ swz(n)) << 4);
    wat[ks] = base + A_BYTES + (is_v * D + mw) * 128 + (((2 * ks + h) ^ wswz(mw)) << 4);
    opaque(aat[ks]);
    opaque(wat[ks]);
  }
  f32x16 acc[MB][2];
  const int steps = heads * STEPS;
  issue(0);
  finish(0);
  for (int i = 0; i < steps; i++) {
    if (i % STEPS == 0) {
#pragma unroll
      for (int b = 0; b < MB; b++) acc[b][0] = acc[b][1] = f32x16{};
    }
    wait_vmcnt<0>();
    __syncthreads();  // the step is whole, and every wave has done with the one before
    if (i + 1 < steps) issue(i + 1);
    const uint32_t st = (i & 1) * STAGE;
#pragma unroll
    for (int ks = 0; ks < 4; ks++) {
      bf16x8 a[MB], x[2];
#pragma unroll
      for (int b = 0; b < MB; b++) a[b] = read_b128(lds_at(wat[ks] + st) + b * 4096);
#pragma unroll
      for (int t = 0; t < 2; t++) x[t] = read_b128(lds_at(aat[ks] + st) + t * 4096);
#pragma unroll
      for (int b = 0; b < MB; b++)
#pragma unroll
        for (int t = 0; t < 2; t++) acc[b][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[b], x[t], acc[b][t], 0, 0, 0);
    }
    if (i + 1 < steps) finish(i + 1);
    if (i % STEPS == STEPS - 1) {
      const int hd = head0 + i / STEPS;
      uint16_t* out = (is_v ? p.vx : p.kx) + ((size_t)hd * p.x_rows + u.x_row + rows0 + n) * D + 16 * h;
#pragma unroll
      for (int t = 0; t < 2; t++) {
        if (rows0 + t * 32 >= u.nrows) continue;  // uniform: rows come in multiples of 64
#pragma unroll
        for (int b = 0; b < MB; b++) {
          uint32_t y[8];
#pragma unroll
          for (int e = 0; e < 8; e++) y[e] = pack_bf16(acc[b][t][2 * e], acc[b][t][2 * e + 1]);
          uint4* dst = (uint4*)(out + (size_t)t * 32 * D + b * 32);
          dst[0] = make_uint4(y[0], y[1], y[2], y[3]);
          dst[1] = make_uint4(y[4], y[5], y[6], y[7]);
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_latent_absorb(const LatentProjParams& p, int64_t n_rows, int latent_dim, int head_dim,
                                hipStream_t stream) {
  if (n_rows <= 0) return hipSuccess;
  const dim3 grid((unsigned)n_rows, p.num_q_heads, latent_dim / kSlice), block(kThreads);
  if (latent_dim == 512) {
    if (head_dim == 128) hipLaunchKernelGGL((latent_absorb_kernel<512, 128>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((latent_absorb_kernel<512, 64>), grid, block, 0, stream, p);
  } else {
    if (head_dim == 128) hipLaunchKernelGGL((latent_absorb_kernel<256, 128>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((latent_absorb_kernel<256, 64>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

hipError_t launch_latent_output(const LatentProjParams& p, int64_t n_rows, int latent_dim, int head_dim,
                                hipStream_t stream) {
  if (n_rows <= 0) return hipSuccess;
  const dim3 grid((unsigned)n_rows, p.num_q_heads), block(kThreads);
  if (latent_dim == 512) {
    if (head_dim == 128) hipLaunchKernelGGL((latent_output_kernel<512, 128>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((latent_output_kernel<512, 64>), grid, block, 0, stream, p);
  } else {
    if (head_dim == 128) hipLaunchKernelGGL((latent_output_kernel<256, 128>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((latent_output_kernel<256, 64>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

template <int LAT, int D>
static void expand_by_type(const LatentExpandParams& p, dim3 grid, bool fp8, hipStream_t stream) {
  if (fp8) hipLaunchKernelGGL((latent_expand_kernel<LAT, D, true>), grid, dim3(kExpThreads), 0, stream, p);
  else hipLaunchKernelGGL((latent_expand_kernel<LAT, D, false>), grid, dim3(kExpThreads), 0, stream, p);
}

hipError_t launch_latent_expand(const LatentExpandParams& p0, int64_t n_units, int latent_dim, int head_dim, bool fp8,
                                hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  LatentExpandParams p = p0;
  // Heads per workgroup: as many as leave at least two workgroups per CU
  p.heads_per = (int32_t)(n_units * p.heads / 512);
  p.heads_per = p.heads_per < 1 ? 1 : (p.heads_per > p.heads ? p.heads : p.heads_per);
  const dim3 grid((unsigned)n_units, (unsigned)((p.heads + p.heads_per - 1) / p.heads_per));
  if (latent_dim == 512) {
    if (head_dim == 128) expand_by_type<512, 128>(p, grid, fp8, stream);
    else expand_by_type<512, 64>(p, grid, fp8, stream);
  } else {
    if (head_dim == 128) expand_by_type<256, 128>(p, grid, fp8, stream);
    else expand_by_type<256, 64>(p, grid, fp8, stream);
  }
  return hipGetLastError();
}

}  // namespace kvx
