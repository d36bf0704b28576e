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
  const LatentRows rows = p.rows[blockIdx.x];
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
  const LatentRows rows = p.rows[blockIdx.x];
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

// Keys and values of 64 cached tokens for every head of the group.
template <int LAT, int D, bool FP8>
__global__ __launch_bounds__(kThreads) void latent_expand_kernel(LatentExpandParams p) {
  using G = LatGeom<LAT>;
  constexpr int NB = 2 * D / 64;  // 16-row blocks of (W_uk, W_uv) per wave
  __shared__ __attribute__((aligned(1024))) uint8_t tile[G::TILE];
  const LatentExpandUnit u = p.units[blockIdx.x];
  const int hd = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
  stage_rows<LAT, FP8, kThreads>(tile, p.pool, p.pool.page_ids + u.page_base, u.key0, u.key_end, u.key_end - 1);
  __syncthreads();
  if (p.rx != nullptr && hd == 0) {
    for (int i = tid; i < kLatTileKeys * 8; i += kThreads) {
      const int r = i / 8, c = i % 8;
      *(uint4*)(p.rx + (size_t)(u.x_row + r) * kLatRope + c * 8) =
          *(const uint4*)(tile + r * G::ROWB + (((LAT / 8 + c) ^ swz(r)) * 16));
    }
  }
  // waves 0 and 1 take W_uk, waves 2 and 3 W_uv
  const bool is_v = wave >= 2;
  const int c0 = (wave & 1) * (D / 2);
  const uint16_t* w = (is_v ? p.w_uv : p.w_uk) + ((size_t)hd * D + c0 + n) * LAT + 8 * g;
  f32x4 acc[4][NB];
#pragma unroll
  for (int kb = 0; kb < 4; kb++)
#pragma unroll
    for (int b = 0; b < NB; b++) acc[kb][b] = f32x4{};
#pragma unroll 4
  for (int ks = 0; ks < LAT / 32; ks++) {
    bf16x8 a[NB];
#pragma unroll
    for (int b = 0; b < NB; b++) a[b] = *(const bf16x8*)(w + (size_t)b * 16 * LAT + ks * 32);
#pragma unroll
    for (int kb = 0; kb < 4; kb++) {
      const int r = kb * 16 + n;
      const bf16x8 x = *(const bf16x8*)(tile + r * G::ROWB + (((ks * 4 + g) ^ swz(r)) * 16));
#pragma unroll
      for (int b = 0; b < NB; b++) acc[kb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[b], x, acc[kb][b], 0, 0, 0);
    }
  }
  uint16_t* out = (is_v ? p.vx : p.kx) + ((size_t)hd * p.x_rows + u.x_row) * D + c0 + 4 * g;
#pragma unroll
  for (int kb = 0; kb < 4; kb++)
#pragma unroll
    for (int b = 0; b < NB; b++) {
      uint2 y;
      y.x = pack_bf16(acc[kb][b][0], acc[kb][b][1]);
      y.y = pack_bf16(acc[kb][b][2], acc[kb][b][3]);
      *(uint2*)(out + (size_t)(kb * 16 + n) * D + b * 16) = y;
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
  if (fp8) hipLaunchKernelGGL((latent_expand_kernel<LAT, D, true>), grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((latent_expand_kernel<LAT, D, false>), grid, dim3(kThreads), 0, stream, p);
}

hipError_t launch_latent_expand(const LatentExpandParams& p, int64_t n_units, int latent_dim, int head_dim, bool fp8,
                                hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  const dim3 grid((unsigned)n_units, p.heads);
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
