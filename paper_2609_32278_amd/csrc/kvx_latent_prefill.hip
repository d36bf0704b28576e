// Attention of per-head queries to expanded keys and values, gfx950.
//
//   o = sum_j w_j v_j / sum_j w_j,   w_j = exp(scale * q . (k_j, r_j)),
// 2 (2 head_dim + 64) operations a visible pair: bound by the matrix unit.  A workgroup takes 256
// tokens of one head, 64 a wave, so that an operand read from LDS feeds two products of 32 x 32;
// queries sit in the accumulator half of the register file, and keys and values of 64 tokens come
// through three LDS stages by direct loads.  The exponentials (as long as a third of the products)
// are formed between the products of the next 32 keys, the loads issued one at a time among them
// (all at once at the start of a tile: calls of 16 turns of 16 heads take 5% more).
// Measured: 8001 tokens of 128 heads in 2.4 ms, 1.1 PFLOP/s (32 tokens a wave, staged through
// registers and with nothing overlapped: 7.4 ms), the matrix unit busy 64 to 68% of the cycles at
// the 2.0 GHz that the power limit leaves.
//
// Roundings: expanded keys and values to bf16 (the products' operands), weights to bf16, the result
// to bf16; scores, sums and reference points are float32.
#include <type_traits>

#include "kvx_latent_tile.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;  // 4 waves x 64 tokens
constexpr int kBN = 64;        // keys per tile
constexpr int kStages = 3;     // tiles in LDS: one attended, one arriving, one being left

// LDS layout of a tile: groups of 8 rows, in a group blocks of 128 bytes of the rows,
// [group][block][8 rows][128 bytes]: K rows are the expanded part and then the shared rotated
// key, V rows follow after the 64 K rows.  A wave-wide direct load of 1 KiB fills a block; the
// 16-byte chunks of a row in a block are stored in the order c ^ order(row), which keeps the
// operand reads (32 rows one chunk; 4 rows four chunks) free of bank conflicts.
__device__ __forceinline__ int order(int r) { return ((r & 2) << 1) | ((r & 4) >> 1) | ((r >> 3) & 1); }

template <int D>
struct PreGeom {
  static constexpr int QK = D + kLatRope;
  static constexpr int KS = QK / 16;   // score product steps
  static constexpr int DB = D / 32;    // 32-dim blocks of the sums
  static constexpr int VB = D / 64;    // blocks of a V row
  static constexpr int KB = VB + 1;    // blocks of a K row
  static constexpr int V0 = 8 * KB * 1024;
  static constexpr int STAGE = V0 + 8 * VB * 1024;
};

template <int D>
__global__ __launch_bounds__(kThreads, 1) void latent_prefill_kernel(LatentPrefillParams p) {
  using G = PreGeom<D>;
  constexpr int AK = 4, AV = 3;  // operand reads ahead of their products
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kStages * G::STAGE];
  const LatentTile u = listed(p, p.units);
  const int ntok = u.head_ntok & 0xFFFF, hd = u.head_ntok >> 16;
  if (ntok == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int Hq = p.num_q_heads;

  const int n_tiles = (u.key_end - u.key_begin + kBN - 1) / kBN;
  // this wave's loads: row groups 2 wave and 2 wave + 1 of a tile
  const uint8_t* kx = (const uint8_t*)(p.kx + ((size_t)hd * p.x_rows + u.x_row + u.key_begin + wave * 16) * D);
  const uint8_t* vx = (const uint8_t*)(p.vx + ((size_t)hd * p.x_rows + u.x_row + u.key_begin + wave * 16) * D);
  const uint8_t* rx = (const uint8_t*)(p.rx + (size_t)(u.x_row + u.key_begin + wave * 16) * kLatRope);
  const int chunk = ((lane & 7) ^ order(lane >> 3)) << 4;
  const int off_x = (lane >> 3) * (D * 2) + chunk, off_r = (lane >> 3) * (kLatRope * 2) + chunk;
  const uint32_t lds0 = lds_address(lds) + wave * (2 * G::KB * 1024), lds0v = lds_address(lds) + G::V0 + wave * (2 * G::VB * 1024);
  constexpr int PIECES = 2 * (G::KB + G::VB);
  size_t aim_at = 0;
  uint32_t aim_stage = 0;
  auto aim = [&](int t) {  // the tile that the next pieces are of
    aim_at = (size_t)(t < n_tiles ? t : n_tiles - 1) * kBN;
    aim_stage = (uint32_t)(t % kStages) * G::STAGE;
  };
  auto piece = [&](int i) {
    const int gr = i / (G::KB + G::VB), j = i % (G::KB + G::VB), flip = gr ? 16 : 0;  // row bit 3 in order
    if (j < G::VB)
      lds_load_1k(kx + (aim_at + gr * 8) * (D * 2) + j * 128, off_x ^ flip, lds0 + aim_stage + (gr * G::KB + j) * 1024);
    else if (j == G::VB)
      lds_load_1k(rx + (aim_at + gr * 8) * (kLatRope * 2), off_r ^ flip, lds0 + aim_stage + (gr * G::KB + j) * 1024);
    else
      lds_load_1k(vx + (aim_at + gr * 8) * (D * 2) + (j - G::KB) * 128, off_x ^ flip,
                  lds0v + aim_stage + (gr * G::VB + j - G::KB) * 1024);
  };

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
    for (int ks = 0; ks < G::KS; ks++) {
      qf[rb][ks] = __builtin_bit_cast(bf16x8, src[ks * 2 + h]);
      keep_in_acc(qf[rb][ks]);
    }
  }
  const int full_end = u.pos0 + 1 < u.key_end ? u.pos0 + 1 : u.key_end;  // keys before it are seen by every row

  f32x16 o[2][G::DB];
  float m[2], ref[2], l[2];
  const float scale = p.scale_log2;
  uint32_t kat[4], vat[2][2];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    kat[i] = lds_address(lds) + (n >> 3) * (G::KB * 1024) + (n & 7) * 128 + (((2 * i + h) ^ order(n)) << 4);
    opaque(kat[i]);
  }
#pragma unroll
  for (int e = 0; e < 2; e++)
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int r = 8 * e + 4 * h + (lane & 15) / 4;
      vat[e][i] = lds_address(lds) + G::V0 + (r >> 3) * (G::VB * 1024) + (r & 7) * 128 +
                  (((4 * i + 2 * (n >> 4) + (lane & 3) / 2) ^ order(r)) << 4) + (lane & 1) * 8;
      opaque(vat[e][i]);
    }

  bf16x8 ka[AK + 1], va[AV + 1];
  // 32 keys at a time: half `kb` of the tile in stage `st`
  auto read_k = [&](uint32_t st, int kb, int ks) {
    return read_b128(lds_at(kat[ks & 3] + st) + (ks >> 2) * 1024 + kb * (4 * G::KB * 1024));
  };
  auto read_v = [&](uint32_t st, int kb, int j) {  // step j: 16 keys (j / DB), dim block j % DB
    const int db = j % G::DB, at = (2 * (2 * kb + j / G::DB)) * (G::VB * 1024) + (db >> 1) * 1024;
    return join(read_tr(lds_at(vat[0][db & 1] + st) + at), read_tr(lds_at(vat[1][db & 1] + st) + at));
  };
  auto start_k = [&](uint32_t st, int kb) {
#pragma unroll
    for (int j = 0; j < AK; j++) ka[j] = read_k(st, kb, j);
  };
  auto start_v = [&](uint32_t st, int kb) {
#pragma unroll
    for (int j = 0; j < AV; j++) va[j] = read_v(st, kb, j);
  };

  uint32_t pk[2][8];  // weights of 32 keys, as pairs
  // The i-th of the 32 scores of a lane (16 of each row): its weight, and pairs packed.
  auto weigh = [&](f32x16 (&s)[2], int i) {
    const int rb = i / 16, e = i % 16;
    s[rb][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][e], scale, -ref[rb]));
    l[rb] += s[rb][e];
    if (e & 1) {
      pk[rb][e / 2] = pack_bf16(s[rb][e - 1], s[rb][e]);
      formed(pk[rb][e / 2]);
      formed(l[rb]);
    }
  };
  // S of 32 keys into `s`, the weights of `w` formed between its steps; START_V: the first V
  // operands of (vst, vkb) are read before the last steps.
  // LOADS: the pieces of a later tile that the value product before left are loaded meanwhile.
  constexpr int VP = PIECES * 2 / 5;  // pieces loaded beside a value product
  auto scores = [&](f32x16 (&s)[2], uint32_t st, int kb, f32x16 (&w)[2], auto weights, auto loads, uint32_t vst,
                    int vkb) {
    constexpr bool W = decltype(weights)::value;
    s[0] = f32x16{};
    s[1] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < G::KS; ks++) {
      if (ks + AK < G::KS) ka[(ks + AK) % (AK + 1)] = read_k(st, kb, ks + AK);
      if (W && ks == G::KS - 3) start_v(vst, vkb);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int rb = 0; rb < 2; rb++) {
        s[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[ks % (AK + 1)], qf[rb][ks], s[rb], 0, 0, 0);
        if constexpr (W) {
#pragma unroll
          for (int i = 0; i < 32; i++)
            if (i * 2 * G::KS / 32 == ks * 2 + rb) weigh(w, i);
        }
      }
      if constexpr (decltype(loads)::value) {
#pragma unroll
        for (int i = VP; i < PIECES; i++)
          if ((i - VP) * G::KS / (PIECES - VP) == ks) piece(i);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto values = [&](uint32_t st, int kb, auto loads) {
#pragma unroll
    for (int j = 0; j < 2 * G::DB; j++) {
      if (j + AV < 2 * G::DB) va[(j + AV) % (AV + 1)] = read_v(st, kb, j + AV);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int rb = 0; rb < 2; rb++) {
        const int half = j / G::DB * 4;
        const bf16x8 b = __builtin_bit_cast(bf16x8, make_uint4(pk[rb][half], pk[rb][half + 1], pk[rb][half + 2], pk[rb][half + 3]));
        o[rb][j % G::DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[j % (AV + 1)], b, o[rb][j % G::DB], 0, 0, 0);
      }
      if constexpr (decltype(loads)::value) {
#pragma unroll
        for (int i = 0; i < VP; i++)
          if (i * 2 * G::DB / VP == j) piece(i);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // accumulator i of a row holds key 8 (i / 4) + 4 h + i % 4 of the 32
  auto mask = [&](f32x16 (&s)[2], int k0) {
#pragma unroll
    for (int rb = 0; rb < 2; rb++)
#pragma unroll
      for (int i = 0; i < 16; i++) s[rb][i] = k0 + 8 * (i / 4) + 4 * h + i % 4 <= limit[rb] ? s[rb][i] : -INFINITY;
  };
  // the reference point moves to the maximum of these scores where that is larger
  auto rereference = [&](f32x16 (&s)[2]) {
#pragma unroll
    for (int rb = 0; rb < 2; rb++) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; i++) mx = fmaxf(mx, s[rb][i]);
      mx *= scale;
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_new = fmaxf(m[rb], mx);
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[rb] - m_new);
      l[rb] *= alpha;
#pragma unroll
      for (int db = 0; db < G::DB; db++) o[rb][db] *= alpha;
      m[rb] = m_new;
      ref[rb] = m_new == -INFINITY ? 0.0f : m_new;
    }
  };

  // One pass over the keys.  FIXED: the reference point stays at the maximum of the first 32.
  auto run = [&](auto fixed) {
    constexpr bool FIXED = decltype(fixed)::value;
#pragma unroll
    for (int rb = 0; rb < 2; rb++) {
      m[rb] = -INFINITY;
      l[rb] = 0.0f;
#pragma unroll
      for (int db = 0; db < G::DB; db++) o[rb][db] = f32x16{};
    }
    using Yes = std::true_type;
    using No = std::false_type;
#pragma unroll
    for (int t = 0; t < 2; t++) {
      aim(t);
#pragma unroll
      for (int i = 0; i < PIECES; i++) piece(i);
    }
    wait_vmcnt<PIECES>();
    __syncthreads();
    f32x16 sa[2], sb[2];
    start_k(0, 0);
    scores(sa, 0, 0, sb, No{}, No{}, 0, 0);
    if (u.key_begin + 32 > full_end) mask(sa, u.key_begin);
    rereference(sa);
    start_k(0, 1);
    uint32_t st = 0;
    for (int t = 0; t < n_tiles; t++) {
      const int k0 = u.key_begin + t * kBN;
      const uint32_t next = st == (kStages - 1) * G::STAGE ? 0 : st + G::STAGE;
      const bool more = t + 1 < n_tiles;
      if constexpr (!FIXED) {
        if (t > 0) rereference(sa);
      }
      scores(sb, st, 1, sa, Yes{}, No{}, st, 0);
      if (k0 + 64 > full_end) mask(sb, k0 + 32);
      // tile t + 1 is whole, and every wave is past tile t - 1, whose stage tile t + 2 takes
      wait_vmcnt<0>();
      __syncthreads();
      aim(t + 2);
      start_k(next, 0);
      values(st, 0, Yes{});
      if constexpr (!FIXED) rereference(sb);
      if (more) {
        scores(sa, next, 0, sb, Yes{}, Yes{}, st, 1);
        if (k0 + 96 > full_end) mask(sa, k0 + 64);
        start_k(next, 1);
      } else {
        start_v(st, 1);
#pragma unroll
        for (int i = 0; i < 32; i++) weigh(sb, i);
      }
      values(st, 1, No{});
      st = next;
    }
    wait_vmcnt<0>();  // pieces past the last tile
    __syncthreads();
  };
  // As in the attention on latents: only where an exponential or a sum overflows float32, or
  // a row sees some of the first 32 keys but no score above -inf there, are the keys gone over
  // again with a reference that moves.
  run(std::true_type{});
  float acc = 0.0f;
#pragma unroll
  for (int rb = 0; rb < 2; rb++) {
    acc += m[rb] == -INFINITY && limit[rb] >= u.key_begin ? INFINITY : l[rb];
#pragma unroll
    for (int db = 0; db < G::DB; db++)
#pragma unroll
      for (int i = 0; i < 16; i++) acc += o[rb][db][i];
  }
  const bool bad = __any(!__builtin_isfinite(acc));
  volatile int* flags = (volatile int*)lds;
  if (lane == 0) flags[wave] = bad;
  __syncthreads();
  const bool again = (flags[0] | flags[1] | flags[2] | flags[3]) != 0;
  __syncthreads();
  if (again) run(std::false_type{});

#pragma unroll
  for (int rb = 0; rb < 2; rb++) {
    const int tok = wave * 64 + rb * 32 + n;
    float lt = l[rb] + __shfl_xor(l[rb], 32, 64);
    if (m[rb] == INFINITY) lt = NAN;  // inf - inf; the weights against such a reference are 0
    const float inv = lt > 0.0f ? 1.0f / lt : (lt == 0.0f ? 0.0f : lt);
    const float lse2 = lt == 0.0f ? -INFINITY : m[rb] + __log2f(lt);
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

// Log-sum-exp combination of a tile's parts; each is read once (25 us for 16 turns of 16 heads).
// Workgroup (merge, 16 or 32 tokens): D / 8 lanes of 8 values per token.
template <int D>
__global__ __launch_bounds__(kThreads) void latent_tile_merge_kernel(LatentTileMergeParams p) {
  constexpr int LPT = D / 8, TPW = kThreads / LPT;
  const LatentTileMerge m = listed(p, p.merges);
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
