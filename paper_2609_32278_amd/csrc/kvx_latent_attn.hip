// Attention of (suffix token, head) rows to the latent cache entries themselves, gfx950.
#include "kvx_latent_tile.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;

template <int LAT, bool FP8, int RB>
__global__ __launch_bounds__(kThreads, 1) void latent_attn_kernel(LatentAttnParams p) {
  using G = LatGeom<LAT>;
  __shared__ __attribute__((aligned(1024))) uint8_t tile[G::TILE];
  __shared__ __attribute__((aligned(16))) uint8_t pl[RB * 16 * 128];
  __shared__ float red[4][RB * 16];
  const LatentUnit u = p.units[blockIdx.x];
  if (u.nrows == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int Hq = p.num_q_heads;
  const int64_t flat0 = (int64_t)u.qo * Hq + u.row0;

  bf16x8 qf[RB][G::KS];
  int limit[RB];  // last visible key of the lane's rows
#pragma unroll
  for (int rb = 0; rb < RB; rb++) {
    const int row = rb * 16 + n;
    const bool valid = row < u.nrows;
    const int pos = u.prefix + (u.row0 + (valid ? row : 0)) / Hq;
    limit[rb] = pos < u.key_end ? pos : u.key_end - 1;
    const uint4* src = (const uint4*)(p.q + (flat0 + (valid ? row : 0)) * G::ROW);
#pragma unroll
    for (int ks = 0; ks < G::KS; ks++) qf[rb][ks] = __builtin_bit_cast(bf16x8, src[ks * 4 + g]);
  }
  const int pos0 = u.prefix + u.row0 / Hq;
  const int safe = pos0 < u.key_begin ? u.key_begin : (pos0 < u.key_end ? pos0 : u.key_end - 1);

  f32x4 o[RB][G::DB];
  float m_run[RB], l_run[RB];
#pragma unroll
  for (int rb = 0; rb < RB; rb++) {
    m_run[rb] = -INFINITY;
    l_run[rb] = 0.0f;
#pragma unroll
    for (int db = 0; db < G::DB; db++) o[rb][db] = f32x4{};
  }

  for (int k0 = u.key_begin; k0 < u.key_end; k0 += kLatTileKeys) {
    __syncthreads();
    stage_rows<LAT, FP8, kThreads>(tile, p.pool, p.pool.page_ids + u.page_base, k0, u.key_end, safe);
    __syncthreads();

    f32x4 s[RB];
#pragma unroll
    for (int rb = 0; rb < RB; rb++) s[rb] = f32x4{};
    const int kr = wave * 16 + n;
#pragma unroll
    for (int ks = 0; ks < G::KS; ks++) {
      const bf16x8 a = *(const bf16x8*)(tile + kr * G::ROWB + (((ks * 4 + g) ^ swz(kr)) * 16));
#pragma unroll
      for (int rb = 0; rb < RB; rb++) s[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[rb][ks], s[rb], 0, 0, 0);
    }
    const int key0 = k0 + wave * 16 + 4 * g;
#pragma unroll
    for (int rb = 0; rb < RB; rb++) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        s[rb][i] = key0 + i <= limit[rb] ? s[rb][i] * p.scale_log2 : -INFINITY;
        mx = fmaxf(mx, s[rb][i]);
      }
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      if (g == 0) red[wave][rb * 16 + n] = mx;
    }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; rb++) {
      const int r = rb * 16 + n;
      const float mt = fmaxf(fmaxf(red[0][r], red[1][r]), fmaxf(red[2][r], red[3][r]));
      const float m_new = fmaxf(m_run[rb], mt);
      const float m = m_new == -INFINITY ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - m);
      m_run[rb] = m_new;
      float pr[4], sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        pr[i] = __builtin_amdgcn_exp2f(s[rb][i] - m);
        sum += pr[i];
      }
      l_run[rb] = l_run[rb] * alpha + sum;
#pragma unroll
      for (int db = 0; db < G::DB; db++) o[rb][db] *= alpha;
      uint2 w;
      w.x = pack_bf16(pr[0], pr[1]);
      w.y = pack_bf16(pr[2], pr[3]);
      *(uint2*)(pl + r * 128 + (((2 * wave + g / 2) ^ (r & 7)) * 16) + (g & 1) * 8) = w;
    }
    __syncthreads();
#pragma unroll
    for (int k2 = 0; k2 < 2; k2++) {
      bf16x8 pb[RB];
#pragma unroll
      for (int rb = 0; rb < RB; rb++) {
        const int r = rb * 16 + n;
        pb[rb] = *(const bf16x8*)(pl + r * 128 + (((4 * k2 + g) ^ (r & 7)) * 16));
      }
#pragma unroll
      for (int db = 0; db < G::DB; db++) {
        s16x4 h[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const int r = k2 * 32 + 8 * g + 4 * e + n / 4;
          const int c = (wave * G::DW + db * 16) / 8 + (n % 4) / 2;
          const uint8_t* at = tile + r * G::ROWB + ((c ^ swz(r)) * 16) + (n % 2) * 8;
          h[e] = read_tr(at);
        }
        const bf16x8 a = join(h[0], h[1]);
#pragma unroll
        for (int rb = 0; rb < RB; rb++)
          o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[rb], o[rb][db], 0, 0, 0);
      }
    }
  }

  __syncthreads();
#pragma unroll
  for (int rb = 0; rb < RB; rb++) {
    float l = l_run[rb];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) red[wave][rb * 16 + n] = l;
  }
  __syncthreads();
#pragma unroll
  for (int rb = 0; rb < RB; rb++) {
    const int r = rb * 16 + n;
    const float l = (red[0][r] + red[1][r]) + (red[2][r] + red[3][r]);
    const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
    const float lse2 = l == 0.0f ? -INFINITY : m_run[rb] + __log2f(l);
    if (u.part < 0) {
      if (r < u.nrows) {
        uint16_t* dst = p.out + (flat0 + r) * LAT + wave * G::DW + 4 * g;
#pragma unroll
        for (int db = 0; db < G::DB; db++) {
          uint2 w;
          w.x = pack_bf16(o[rb][db][0] * inv, o[rb][db][1] * inv);
          w.y = pack_bf16(o[rb][db][2] * inv, o[rb][db][3] * inv);
          *(uint2*)(dst + db * 16) = w;
        }
        if (p.lse != nullptr && wave == 0 && g == 0) p.lse[flat0 + r] = lse2 * kLn2;
      }
    } else {
      float* dst = p.o_part + (size_t)u.part * (RB * 16 * LAT) + (size_t)((wave * RB + rb) * G::DB) * 256 + lane * 4;
#pragma unroll
      for (int db = 0; db < G::DB; db++) *(f32x4*)(dst + db * 256) = o[rb][db] * inv;
      if (wave == 0 && g == 0) p.lse_part[(size_t)u.part * (RB * 16) + r] = lse2;
    }
  }
}

// Log-sum-exp combination of a tile's parts: workgroup (merge, row block), lanes as above.
template <int LAT, int RB>
__global__ __launch_bounds__(kThreads) void latent_merge_kernel(LatentMergeParams p) {
  using G = LatGeom<LAT>;
  const LatentMerge m = p.merges[blockIdx.x];
  const int rb = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const int r = rb * 16 + n;
  if (rb * 16 >= m.nrows) return;
  float top = -INFINITY;
  for (int i = 0; i < m.nparts; i++)
    top = fmaxf(top, p.lse_part[(size_t)(m.part0 + i) * (RB * 16) + r]);
  const float ref = top == -INFINITY ? 0.0f : top;
  f32x4 o[G::DB];
#pragma unroll
  for (int db = 0; db < G::DB; db++) o[db] = f32x4{};
  float total = 0.0f;
  for (int i = 0; i < m.nparts; i++) {
    const size_t part = (size_t)(m.part0 + i);
    const float w = __builtin_amdgcn_exp2f(p.lse_part[part * (RB * 16) + r] - ref);
    total += w;
    const float* src = p.o_part + part * (RB * 16 * LAT) + (size_t)((wave * RB + rb) * G::DB) * 256 + lane * 4;
#pragma unroll
    for (int db = 0; db < G::DB; db++) o[db] += *(const f32x4*)(src + db * 256) * w;
  }
  if (r >= m.nrows) return;
  const float inv = total > 0.0f ? 1.0f / total : (total == 0.0f ? 0.0f : total);
  const int64_t flat = (int64_t)m.qo * p.num_q_heads + m.row0 + r;
  uint16_t* dst = p.out + flat * LAT + wave * G::DW + 4 * g;
#pragma unroll
  for (int db = 0; db < G::DB; db++) {
    uint2 w;
    w.x = pack_bf16(o[db][0] * inv, o[db][1] * inv);
    w.y = pack_bf16(o[db][2] * inv, o[db][3] * inv);
    *(uint2*)(dst + db * 16) = w;
  }
  if (p.lse != nullptr && wave == 0 && g == 0) p.lse[flat] = (ref + __log2f(total)) * kLn2;
}

template <int LAT, bool FP8>
void attn_by_blocks(const LatentAttnParams& p, unsigned n, int rb, hipStream_t s) {
  if (rb == 1) hipLaunchKernelGGL((latent_attn_kernel<LAT, FP8, 1>), dim3(n), dim3(kThreads), 0, s, p);
  else if (rb == 2) hipLaunchKernelGGL((latent_attn_kernel<LAT, FP8, 2>), dim3(n), dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((latent_attn_kernel<LAT, FP8, 4>), dim3(n), dim3(kThreads), 0, s, p);
}

template <int LAT>
void merge_by_blocks(const LatentMergeParams& p, unsigned n, int rb, hipStream_t s) {
  if (rb == 1) hipLaunchKernelGGL((latent_merge_kernel<LAT, 1>), dim3(n, 1), dim3(kThreads), 0, s, p);
  else if (rb == 2) hipLaunchKernelGGL((latent_merge_kernel<LAT, 2>), dim3(n, 2), dim3(kThreads), 0, s, p);
  else hipLaunchKernelGGL((latent_merge_kernel<LAT, 4>), dim3(n, 4), dim3(kThreads), 0, s, p);
}

}  // namespace

hipError_t launch_latent_attention(const LatentAttnParams& p, int64_t n_units, int latent_dim, bool fp8, int row_blocks,
                                   hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  const unsigned n = (unsigned)n_units;
  if (latent_dim == 512) {
    if (fp8) attn_by_blocks<512, true>(p, n, row_blocks, stream);
    else attn_by_blocks<512, false>(p, n, row_blocks, stream);
  } else {
    if (fp8) attn_by_blocks<256, true>(p, n, row_blocks, stream);
    else attn_by_blocks<256, false>(p, n, row_blocks, stream);
  }
  return hipGetLastError();
}

hipError_t launch_latent_merge(const LatentMergeParams& p, int64_t n_merges, int latent_dim, int row_blocks,
                               hipStream_t stream) {
  if (n_merges <= 0) return hipSuccess;
  if (latent_dim == 512) merge_by_blocks<512>(p, (unsigned)n_merges, row_blocks, stream);
  else merge_by_blocks<256>(p, (unsigned)n_merges, row_blocks, stream);
  return hipGetLastError();
}

}  // namespace kvx
