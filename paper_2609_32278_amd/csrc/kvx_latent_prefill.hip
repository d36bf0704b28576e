// Attention of per-head queries to expanded keys and values, gfx950.
#include "kvx_latent_tile.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;  // 4 waves x 64 tokens
constexpr int kBN = 64;

template <int D>
struct PreGeom {
  static constexpr int QK = D + kLatRope;
  static constexpr int KS = QK / 16;
  static constexpr int DB = D / 32;
  static constexpr int KROWB = QK * 2;
  static constexpr int VROWB = D * 2;
};

// Stored chunk of chunk c of a row.  K rows of 384 bytes are 32 banks apart modulo 64, those
// of 256 bytes none; V rows of 256 bytes none, those of 128 bytes 32.
template <int D>
__device__ __forceinline__ int kswz(int r) {
  if constexpr (D == 128) return swz(r);
  else return r & 15;
}
template <int D>
__device__ __forceinline__ int vswz(int r) {
  if constexpr (D == 128) return ((r & 3) << 1) | ((r >> 2) & 1) | (r & 8);
  else return (r & 2) | (r & 4) | ((r >> 3) & 1);
}

template <int D>
__global__ __launch_bounds__(kThreads, 1) void latent_prefill_kernel(LatentPrefillParams p) {
  using G = PreGeom<D>;
  __shared__ __attribute__((aligned(1024))) uint8_t kl[kBN * G::KROWB];
  __shared__ __attribute__((aligned(1024))) uint8_t vl[kBN * G::VROWB];
  const LatentTile u = p.units[blockIdx.x];
  const int ntok = u.head_ntok & 0xFFFF, hd = u.head_ntok >> 16;
  if (ntok == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int Hq = p.num_q_heads;
  bf16x8 qf[2][G::KS];
  int limit[2];
  int64_t flat[2];
#pragma unroll
  for (int rb = 0; rb < 2; rb++) {
    const int tok = wave * 64 + rb * 32 + n, t = tok < ntok ? tok : 0;
    flat[rb] = (int64_t)(u.qo_row + t) * Hq + p.head0 + hd;
    limit[rb] = u.pos0 + t < u.key_end ? u.pos0 + t : u.key_end - 1;
    const uint4* src = (const uint4*)(p.q + flat[rb] * G::QK);
#pragma unroll
    for (int ks = 0; ks < G::KS; ks++) qf[rb][ks] = __builtin_bit_cast(bf16x8, src[ks * 2 + h]);
  }
  const uint16_t* kx = p.kx + ((size_t)hd * p.x_rows + u.x_row) * D;
  const uint16_t* vx = p.vx + ((size_t)hd * p.x_rows + u.x_row) * D;
  const uint16_t* rx = p.rx + (size_t)u.x_row * kLatRope;
  f32x16 o[2][G::DB];
  float m_run[2], l_run[2];
#pragma unroll
  for (int rb = 0; rb < 2; rb++) {
    m_run[rb] = -INFINITY;
    l_run[rb] = 0.0f;
#pragma unroll
    for (int db = 0; db < G::DB; db++) o[rb][db] = f32x16{};
  }
  for (int k0 = u.key_begin; k0 < u.key_end; k0 += kBN) {
    __syncthreads();
    for (int i = tid; i < kBN * (D / 8); i += kThreads) {
      const int r = i / (D / 8), c = i % (D / 8);
      *(uint4*)(kl + r * G::KROWB + ((c ^ kswz<D>(r)) * 16)) = *(const uint4*)(kx + (size_t)(k0 + r) * D + c * 8);
      *(uint4*)(vl + r * G::VROWB + ((c ^ vswz<D>(r)) * 16)) = *(const uint4*)(vx + (size_t)(k0 + r) * D + c * 8);
    }
    for (int i = tid; i < kBN * 8; i += kThreads) {
      const int r = i / 8, c = i % 8;
      *(uint4*)(kl + r * G::KROWB + (((D / 8 + c) ^ kswz<D>(r)) * 16)) =
          *(const uint4*)(rx + (size_t)(k0 + r) * kLatRope + c * 8);
    }
    __syncthreads();
    f32x16 s[2][2];  // [row block][key block]
#pragma unroll
    for (int rb = 0; rb < 2; rb++) s[rb][0] = s[rb][1] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < G::KS; ks++)
#pragma unroll
      for (int kb = 0; kb < 2; kb++) {
        const int r = kb * 32 + n;
        const bf16x8 a = *(const bf16x8*)(kl + r * G::KROWB + (((ks * 2 + h) ^ kswz<D>(r)) * 16));
#pragma unroll
        for (int rb = 0; rb < 2; rb++)
          s[rb][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[rb][ks], s[rb][kb], 0, 0, 0);
      }
    // accumulator i of a key block holds key 8 (i / 4) + 4 h + i % 4 of it
    bf16x8 pb[2][4];
#pragma unroll
    for (int rb = 0; rb < 2; rb++) {
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; kb++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
          const int key = k0 + kb * 32 + 8 * (i / 4) + 4 * h + i % 4;
          const float x = key <= limit[rb] ? s[rb][kb][i] * p.scale_log2 : -INFINITY;
          s[rb][kb][i] = x;
          mx = fmaxf(mx, x);
        }
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_new = fmaxf(m_run[rb], mx), m = m_new == -INFINITY ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - m);
      m_run[rb] = m_new;
      float sum = 0.0f;
#pragma unroll
      for (int kb = 0; kb < 2; kb++)
#pragma unroll
        for (int half = 0; half < 2; half++) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const float a = __builtin_amdgcn_exp2f(s[rb][kb][8 * half + 2 * e] - m);
            const float b = __builtin_amdgcn_exp2f(s[rb][kb][8 * half + 2 * e + 1] - m);
            sum += a + b;
            w[e] = pack_bf16(a, b);
          }
          pb[rb][2 * kb + half] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
        }
      l_run[rb] = l_run[rb] * alpha + sum;
#pragma unroll
      for (int db = 0; db < G::DB; db++) o[rb][db] *= alpha;
    }
    // 16 keys a step: slot (h, j) of the step is key 8 (j / 4) + 4 h + j % 4, as P has them
#pragma unroll
    for (int st = 0; st < 4; st++)
#pragma unroll
      for (int db = 0; db < G::DB; db++) {
        s16x4 v[2];
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const int r = st * 16 + 8 * e + 4 * h + (lane & 15) / 4;
          const int c = (db * 32 + (n & 16)) / 8 + (lane & 3) / 2;
          v[e] = read_tr(vl + r * G::VROWB + ((c ^ vswz<D>(r)) * 16) + (lane & 1) * 8);
        }
        const bf16x8 a = join(v[0], v[1]);
#pragma unroll
        for (int rb = 0; rb < 2; rb++)
          o[rb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[rb][st], o[rb][db], 0, 0, 0);
      }
  }
#pragma unroll
  for (int rb = 0; rb < 2; rb++) {
    const int tok = wave * 64 + rb * 32 + n;
    const float l = l_run[rb] + __shfl_xor(l_run[rb], 32, 64);
    const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
    const float lse2 = l == 0.0f ? -INFINITY : m_run[rb] + __log2f(l);
    if (tok >= ntok) continue;
    if (u.part < 0) {
      uint16_t* dst = p.out + flat[rb] * D + 4 * h;
#pragma unroll
      for (int db = 0; db < G::DB; db++)
#pragma unroll
        for (int i4 = 0; i4 < 4; i4++) {
          uint2 w;
          w.x = pack_bf16(o[rb][db][4 * i4] * inv, o[rb][db][4 * i4 + 1] * inv);
          w.y = pack_bf16(o[rb][db][4 * i4 + 2] * inv, o[rb][db][4 * i4 + 3] * inv);
          *(uint2*)(dst + db * 32 + 8 * i4) = w;
        }
      if (p.lse != nullptr && h == 0) p.lse[flat[rb]] = lse2 * kLn2;
    } else {
      float* dst = p.o_part + ((size_t)u.part * kLatTileTok + tok) * D + 4 * h;
#pragma unroll
      for (int db = 0; db < G::DB; db++)
#pragma unroll
        for (int i4 = 0; i4 < 4; i4++) {
          f32x4 w;
#pragma unroll
          for (int e = 0; e < 4; e++) w[e] = o[rb][db][4 * i4 + e] * inv;
          *(f32x4*)(dst + db * 32 + 8 * i4) = w;
        }
      if (h == 0) p.lse_part[(size_t)u.part * kLatTileTok + tok] = lse2;
    }
  }
}

// Workgroup (merge, 16 tokens): D / 8 lanes of 8 values per token.
template <int D>
__global__ __launch_bounds__(kThreads) void latent_tile_merge_kernel(LatentTileMergeParams p) {
  constexpr int LPT = D / 8, TPW = kThreads / LPT;
  const LatentTileMerge m = p.merges[blockIdx.x];
  const int tok = blockIdx.y * TPW + threadIdx.x / LPT, c = threadIdx.x % LPT;
  if (tok >= (m.head_ntok & 0xFFFF)) return;
  float top = -INFINITY;
  for (int i = 0; i < m.nparts; i++) top = fmaxf(top, p.lse_part[(size_t)(m.part0 + i) * kLatTileTok + tok]);
  const float ref = top == -INFINITY ? 0.0f : top;
  f32x4 a{}, b{};
  float total = 0.0f;
  for (int i = 0; i < m.nparts; i++) {
    const size_t at = (size_t)(m.part0 + i) * kLatTileTok + tok;
    const float w = __builtin_amdgcn_exp2f(p.lse_part[at] - ref);
    total += w;
    const f32x4* src = (const f32x4*)(p.o_part + at * D + c * 8);
    a += src[0] * w;
    b += src[1] * w;
  }
  const float inv = total > 0.0f ? 1.0f / total : (total == 0.0f ? 0.0f : total);
  const int64_t flat = (int64_t)(m.qo_row + tok) * p.num_q_heads + p.head0 + (m.head_ntok >> 16);
  *(uint4*)(p.out + flat * D + c * 8) = make_uint4(pack_bf16(a[0] * inv, a[1] * inv), pack_bf16(a[2] * inv, a[3] * inv),
                                                   pack_bf16(b[0] * inv, b[1] * inv), pack_bf16(b[2] * inv, b[3] * inv));
  if (p.lse != nullptr && c == 0) p.lse[flat] = (ref + __log2f(total)) * kLn2;
}

}  // namespace

hipError_t launch_latent_prefill(const LatentPrefillParams& p, int64_t n_units, int head_dim, hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  const dim3 grid((unsigned)n_units), block(kThreads);
  if (head_dim == 128) hipLaunchKernelGGL((latent_prefill_kernel<128>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((latent_prefill_kernel<64>), grid, block, 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_latent_tile_merge(const LatentTileMergeParams& p, int64_t n_merges, int head_dim,
                                    hipStream_t stream) {
  if (n_merges <= 0) return hipSuccess;
  const dim3 grid((unsigned)n_merges, kLatTileTok / (kThreads / (head_dim / 8))), block(kThreads);
  if (head_dim == 128) hipLaunchKernelGGL((latent_tile_merge_kernel<128>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((latent_tile_merge_kernel<64>), grid, block, 0, stream, p);
  return hipGetLastError();
}

}  // namespace kvx
