// Stores into a page-scaled pool, and tokens read back from any pool, gfx950 (CDNA4).
//
// A page-scaled pool holds e4m3 codes, and for every page and KV head one power of two for K and
// one for V: the smallest 2^e with max|x| <= 448 * 2^e over the values that the page then holds,
// e in [-117, 119].  e4m3 has its own exponent, so a power of two loses nothing against a finer
// scale but where values fall below 2^-6 of it, and the attention gets it for nothing: the
// conversion of two codes to bf16 takes a power of two, and code * 2^e is a bf16 value exactly.
//
// A store writes whole pages: a first page that keeps tokens from before (as it holds them) takes
// them into its maximum and rounds them again if the scale moved; slots past the last token
// become zero.  What a page holds thus follows from its live values alone, never from what
// was in it before they came.
//
// HBM bound: every row is read once and every code written once.  A wave takes one (page,
// head) block of K or of V (two of head_dim 64): four 16-byte loads a lane in flight, the maximum
// over its lanes, no barrier.  K rows go out as they lie; for V a lane takes four slots that
// follow each other, so that the conversion packs them into a word of the pool's [dim][16 slots]
// order, and the wave's words meet in LDS to leave as 16-byte pieces.  18155 tokens of 8 heads of 128
// dims: the store takes 20.9 us (5.3 TB/s), their way back 18.9 (5.9 TB/s).

#include "kvx_internal.h"
#include "kvx_rope_util.h"
#include "kvx_store_util.h"

namespace kvx {
namespace {

enum PageStoreMode { kPageStorePlain, kPageStoreHalf, kPageStoreInterleaved };

// How a wave's lanes lie over the (page, head) blocks it takes.
template <int D>
struct BlockLanes {
  static constexpr int CPR = D / 8;      // lanes of a row, 8 dims each
  static constexpr int LANES = 4 * CPR;  // of a block
  static constexpr int BLOCKS = 64 / LANES;
  int sub, c, q;  // block of the wave; 8-dim chunk; a quarter of the slots
  __device__ __forceinline__ BlockLanes() {
    const int lane = threadIdx.x & 63;
    sub = lane / LANES;
    c = lane % CPR;
    q = lane / CPR % 4;
  }
};

// Words of V codes in LDS: [chunk c of the wave][dim e of it][slot quarter], chunks padded so that
// the lanes' words (same e) fall on all banks.
constexpr int kChunkWords = 36;
// ... of bf16 values: two words a slot quarter
constexpr int kChunkWords16 = 72;

// LDS of one wave: its writes before, its reads after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Four codes -> floats times a power of two (exact)
__device__ __forceinline__ void codes_to_f32(uint32_t w, float by, float (&x)[4]) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * by;
  x[1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * by;
  x[2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * by;
  x[3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * by;
}

// The block's exponent, from its lanes' values.  NaN counts for nothing (fmaxf).
template <int D>
__device__ __forceinline__ int block_exp(const float (&x)[4][8]) {
  float amax = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; j++)
#pragma unroll
    for (int e = 0; e < 8; e++) amax = fmaxf(amax, fabsf(x[j][e]));
#pragma unroll
  for (int m = 1; m < BlockLanes<D>::LANES; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m, 64));
  return scale_exp(amax);
}

// Grid: x = the unit (a touched page); y = groups of 1 << p.lg_q Q heads, then groups of K heads,
// then of V heads, one wave for each BLOCKS of them.
template <int D, PageStoreMode MODE>
__global__ __launch_bounds__(kStoreThreads) void store_kv_page_kernel(RopeParams p) {
  using L = BlockLanes<D>;
  constexpr bool ROPE = MODE != kPageStorePlain, INTERLEAVED = MODE == kPageStoreInterleaved;
  union Shared {
    float2 cs[ROPE ? kPageSize : 1][kRopeMaxPlanes];        // (cos, sin) of every live slot and plane
    uint32_t vt[kStoreThreads / 64][16 * kChunkWords];      // V codes of each wave
  };
  __shared__ __attribute__((aligned(16))) Shared sm;
  const RopeUnit u = p.reqs.n > 0 ? inline_unit(p.reqs, blockIdx.x) : p.units[blockIdx.x];
  const int H = p.num_kv_heads;
  int y = blockIdx.y;
  if constexpr (ROPE) {
    const int Hq = p.num_q_heads, q_groups = (Hq + (1 << p.lg_q) - 1) >> p.lg_q;
    if (y < q_groups) {
      const int h0 = y << p.lg_q, nh = Hq - h0 < (1 << p.lg_q) ? Hq - h0 : 1 << p.lg_q;
      const int64_t row0 = (int64_t)u.row_slot0 + u.slot_begin;
      uint16_t* qo = p.q_out + row0 * Hq * D;
      auto angles = [&]() {
        fill_angles(sm.cs, u, p.rotary_dim, p.rev_freq);
        __syncthreads();
      };
      rope_rows<D, INTERLEAVED>(p.q + row0 * Hq * D, u.slot_end - u.slot_begin, Hq, h0, nh, p.lg_q, u.slot_begin,
                                sm.cs, p.q_norm, p.norm_eps, p.rotary_dim, angles,
                                [&](int tok, int hd, int cc, const float(&v)[8]) {
                                  store16<true>(qo + ((size_t)tok * Hq + hd) * D + cc * 8, pack_bf16x8(v));
                                });
      return;
    }
    y -= q_groups;
  }
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, per = waves * L::BLOCKS;  // heads per workgroup
  const int groups = (H + per - 1) / per;
  const bool is_v = y >= groups;  // uniform
  const L l;
  const int hd = (is_v ? y - groups : y) * per + wave * L::BLOCKS + l.sub;
  const bool in = hd < H;
  const int64_t entry = (int64_t)p.page_ids[u.page_pos] * H + (in ? hd : 0);
  uint8_t* block = (uint8_t*)(is_v ? p.v_pool : p.k_pool) + entry * (kPageSize * D);
  float* scale = p.page_scale + 2 * entry + (is_v ? 1 : 0);
  // the slots of this lane's four rows
  const int s0 = is_v ? 4 * l.q : l.q, step = is_v ? 1 : 4;
  const uint16_t* src = (is_v ? p.v_ext : p.k_ext) + ((int64_t)u.row_slot0 * H + hd) * D + l.c * 8;

  uint4 raw[4];
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const int slot = s0 + step * j;
    raw[j] = make_uint4(0, 0, 0, 0);
    if (in && slot >= u.slot_begin && slot < u.slot_end) raw[j] = *(const uint4*)(src + (int64_t)slot * H * D);
  }
  float x[4][8];
#pragma unroll
  for (int j = 0; j < 4; j++) unpack_bf16x8(raw[j], x[j]);

  if constexpr (ROPE) {
    fill_angles(sm.cs, u, p.rotary_dim, p.rev_freq);
    __syncthreads();
    if (!is_v) {
      const RopeLane<D, INTERLEAVED> rl(p.rotary_dim);
      float w[8];
      if (p.k_norm) unpack_bf16x8(*(const uint4*)(p.k_norm + l.c * 8), w);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        if (p.k_norm) {  // uniform
          float ss = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; e++) ss = fmaf(x[j][e], x[j][e], ss);
#pragma unroll
          for (int m = 1; m < L::CPR; m <<= 1) ss += __shfl_xor(ss, m, 64);
          const float inv = 1.0f / sqrtf(ss * (1.0f / D) + p.norm_eps);
#pragma unroll
          for (int e = 0; e < 8; e++) x[j][e] = (x[j][e] * inv) * w[e];
        }
        const int slot = s0 + step * j;
        rope_chunk<D, INTERLEAVED>(x[j], rl, sm.cs[slot]);
        if (slot < u.slot_begin || slot >= u.slot_end) {  // no such token: its angles are not there either
#pragma unroll
          for (int e = 0; e < 8; e++) x[j][e] = 0.0f;
        }
      }
    }
  }

  if (u.slot_begin > 0) {  // uniform: tokens from before, as the page holds them
    const float by = *scale;
    if (is_v) {
#pragma unroll
      for (int e = 0; e < 8; e++) {
        float o[4];
        codes_to_f32(*(const uint32_t*)(block + (8 * l.c + e) * kPageSize + 4 * l.q), by, o);
#pragma unroll
        for (int j = 0; j < 4; j++)
          if (s0 + j < u.slot_begin) x[j][e] = o[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int slot = s0 + step * j;
        if (slot >= u.slot_begin) continue;
        const uint2 w = *(const uint2*)(block + slot * D + 8 * l.c);
        float o[4];
        codes_to_f32(w.x, by, o);
#pragma unroll
        for (int e = 0; e < 4; e++) x[j][e] = o[e];
        codes_to_f32(w.y, by, o);
#pragma unroll
        for (int e = 0; e < 4; e++) x[j][4 + e] = o[e];
      }
    }
  }

  const int ex = block_exp<D>(x);
  const float by = __uint_as_float((uint32_t)(127 - ex) << 23);
  if (in && l.c == 0 && l.q == 0) *scale = __uint_as_float((uint32_t)(127 + ex) << 23);
  if (!is_v) {
    if (!in) return;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      uint2 code;
      code.x = codes4(x[j][0] * by, x[j][1] * by, x[j][2] * by, x[j][3] * by);
      code.y = codes4(x[j][4] * by, x[j][5] * by, x[j][6] * by, x[j][7] * by);
      *(uint2*)(block + (s0 + step * j) * D + 8 * l.c) = code;
    }
    return;
  }
  if constexpr (ROPE) __syncthreads();  // the angles have been read; uniform: a workgroup is all K or all V
  uint32_t* vt = sm.vt[wave];
#pragma unroll
  for (int e = 0; e < 8; e++)
    vt[(l.sub * L::CPR + l.c) * kChunkWords + 4 * e + l.q] =
        codes4(x[0][e] * by, x[1][e] * by, x[2][e] * by, x[3][e] * by);
  wave_sync();
  const int lane_of_block = threadIdx.x & (L::LANES - 1);
#pragma unroll
  for (int k = 0; k < 2; k++) {
    const int d = lane_of_block + L::LANES * k;
    const uint4 w = *(const uint4*)&vt[(l.sub * L::CPR + d / 8) * kChunkWords + 4 * (d % 8)];
    if (in) *(uint4*)(block + d * kPageSize) = w;
  }
}

// 8 codes -> 8 bf16 values, times a power of two (exact)
__device__ __forceinline__ uint4 dequant_pow2(uint2 c, float by) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, by, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, by, true)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, by, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, by, true)));
}
// ... times any scale, rounded once
__device__ __forceinline__ uint4 dequant(uint2 c, float by) {
  float lo[4], hi[4];
  codes_to_f32(c.x, by, lo);
  codes_to_f32(c.y, by, hi);
  const float y[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return pack_bf16x8(y);
}

// Bytes j of four words -> word j
__device__ __forceinline__ void transpose4x4(const uint32_t (&w)[4], uint32_t (&t)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  t[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
  t[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
  t[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
  t[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

// Tokens of a page as bf16 rows, the store's way back: grid and lanes as there.
template <int D, int KIND>
__global__ __launch_bounds__(kStoreThreads) void load_kv_kernel(LoadParams p) {
  using L = BlockLanes<D>;
  constexpr bool BF16 = KIND == KVX_KV_BF16;
  constexpr int EB = BF16 ? 2 : 1, WORDS = BF16 ? kChunkWords16 : kChunkWords;
  __shared__ __attribute__((aligned(16))) uint32_t sm[kStoreThreads / 64][16 * WORDS];
  const RopeUnit u = p.reqs.n > 0 ? inline_unit(p.reqs, blockIdx.x) : p.units[blockIdx.x];
  const int H = p.num_kv_heads, y = blockIdx.y;
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, per = waves * L::BLOCKS;
  const int groups = (H + per - 1) / per;
  const bool is_v = y >= groups;  // uniform
  const L l;
  const int hd = (is_v ? y - groups : y) * per + wave * L::BLOCKS + l.sub;
  if (hd >= H) return;  // whole blocks of lanes; what they share with others is nothing
  const int64_t entry = (int64_t)p.page_ids[u.page_pos] * H + hd;
  const uint8_t* block = (const uint8_t*)(is_v ? p.v_pool : p.k_pool) + entry * (kPageSize * D * EB);
  uint16_t* dst = (is_v ? p.v_out : p.k_out) + ((int64_t)u.row_slot0 * H + hd) * D + l.c * 8;
  float by = 1.0f;
  if constexpr (KIND == KVX_KV_FP8_PAGE) by = p.page_scale[2 * entry + (is_v ? 1 : 0)];
  if constexpr (KIND == KVX_KV_FP8_E4M3) by = (is_v ? p.v_scale : p.k_scale)[hd];
  auto value = [&](uint2 c) {
    if constexpr (KIND == KVX_KV_FP8_PAGE) return dequant_pow2(c, by);
    else return dequant(c, by);
  };
  auto put = [&](int slot, uint4 row) {
    if (slot >= u.slot_begin && slot < u.slot_end) *(uint4*)(dst + (int64_t)slot * H * D) = row;
  };
  if (!is_v) {
    if constexpr (BF16) {
      uint4 w[4];
#pragma unroll
      for (int j = 0; j < 4; j++) w[j] = load16<true>(block + ((4 * j + l.q) * D + 8 * l.c) * 2);
#pragma unroll
      for (int j = 0; j < 4; j++) put(4 * j + l.q, w[j]);
    } else {
      uint2 w[4];
#pragma unroll
      for (int j = 0; j < 4; j++) w[j] = *(const uint2*)(block + (4 * j + l.q) * D + 8 * l.c);
#pragma unroll
      for (int j = 0; j < 4; j++) put(4 * j + l.q, value(w[j]));
    }
    return;
  }
  uint32_t* vt = sm[wave];
  const int lane_of_block = threadIdx.x & (L::LANES - 1);
  // [dim][16 slots] in 16-byte pieces
  constexpr int PIECES = 2 * EB;
  uint4 piece[PIECES];
#pragma unroll
  for (int k = 0; k < PIECES; k++) piece[k] = load16<true>(block + (lane_of_block + L::LANES * k) * 16);
#pragma unroll
  for (int k = 0; k < PIECES; k++) {
    const int i = lane_of_block + L::LANES * k, d = i / EB;
    *(uint4*)&vt[(l.sub * L::CPR + d / 8) * WORDS + 4 * EB * (d % 8) + 4 * (i % EB)] = piece[k];
  }
  wave_sync();
  const uint32_t* from = vt + (l.sub * L::CPR + l.c) * WORDS;
  if constexpr (BF16) {
    uint2 w[8];
#pragma unroll
    for (int e = 0; e < 8; e++) w[e] = *(const uint2*)(from + 8 * e + 2 * l.q);
    uint32_t row[4][4];
#pragma unroll
    for (int i = 0; i < 4; i++) {  // dims 2 i, 2 i + 1 of the chunk
      row[0][i] = __builtin_amdgcn_perm(w[2 * i + 1].x, w[2 * i].x, 0x05040100);
      row[1][i] = __builtin_amdgcn_perm(w[2 * i + 1].x, w[2 * i].x, 0x07060302);
      row[2][i] = __builtin_amdgcn_perm(w[2 * i + 1].y, w[2 * i].y, 0x05040100);
      row[3][i] = __builtin_amdgcn_perm(w[2 * i + 1].y, w[2 * i].y, 0x07060302);
    }
#pragma unroll
    for (int j = 0; j < 4; j++) put(4 * l.q + j, make_uint4(row[j][0], row[j][1], row[j][2], row[j][3]));
  } else {
    uint32_t a[4], b[4], ta[4], tb[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
      a[e] = from[4 * e + l.q];
      b[e] = from[4 * (4 + e) + l.q];
    }
    transpose4x4(a, ta);
    transpose4x4(b, tb);
#pragma unroll
    for (int j = 0; j < 4; j++) put(4 * l.q + j, value(make_uint2(ta[j], tb[j])));
  }
}

// Waves of a workgroup whose heads (K or V) are `heads`, and the workgroups of a page.
struct HeadGrid {
  unsigned threads, groups;
};
HeadGrid head_grid(int heads, int head_dim, bool full) {
  const int per_wave = 128 / head_dim, need = (heads + per_wave - 1) / per_wave;
  const int waves = full || need > kStoreThreads / 64 ? kStoreThreads / 64 : need;
  return {64u * (unsigned)waves, 2u * (unsigned)((need + waves - 1) / waves)};
}

template <int D>
void launch_store_for(const RopeParams& p, dim3 grid, dim3 block, PageStoreMode mode, hipStream_t stream) {
  if (mode == kPageStorePlain) hipLaunchKernelGGL((store_kv_page_kernel<D, kPageStorePlain>), grid, block, 0, stream, p);
  else if (mode == kPageStoreHalf) hipLaunchKernelGGL((store_kv_page_kernel<D, kPageStoreHalf>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((store_kv_page_kernel<D, kPageStoreInterleaved>), grid, block, 0, stream, p);
}

template <int D>
void launch_load_for(const LoadParams& p, dim3 grid, dim3 block, int32_t kind, hipStream_t stream) {
  if (kind == KVX_KV_BF16) hipLaunchKernelGGL((load_kv_kernel<D, KVX_KV_BF16>), grid, block, 0, stream, p);
  else if (kind == KVX_KV_FP8_E4M3) hipLaunchKernelGGL((load_kv_kernel<D, KVX_KV_FP8_E4M3>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((load_kv_kernel<D, KVX_KV_FP8_PAGE>), grid, block, 0, stream, p);
}

}  // namespace

hipError_t launch_store_kv_page(const RopeParams& p0, int64_t n_units, int head_dim, bool interleaved,
                                hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  RopeParams p = p0;
  const PageStoreMode mode = p.rotary_dim == 0 ? kPageStorePlain : interleaved ? kPageStoreInterleaved : kPageStoreHalf;
  const HeadGrid kv = head_grid(p.num_kv_heads, head_dim, mode != kPageStorePlain);
  int64_t q_groups = 0;
  p.lg_q = 0;
  if (mode != kPageStorePlain && p.num_q_heads > 0) {
    // as in the rotating store of the other pools: 4 Q heads a workgroup, more once there are
    // 2048 of them, never above 16 but for the grid's bound
    int lg_all = 0;
    while ((1 << lg_all) < p.num_q_heads) lg_all++;
    for (int lg = 2;; lg++) {
      p.lg_q = lg < lg_all ? lg : lg_all;
      q_groups = ((int64_t)p.num_q_heads + (1 << p.lg_q) - 1) >> p.lg_q;
      const int64_t groups = q_groups + kv.groups;
      if (groups <= 65535 && (lg >= 4 || n_units * groups <= 2048)) break;
    }
  }
  const dim3 grid((unsigned)n_units, (unsigned)q_groups + kv.groups), block(kv.threads);
  if (head_dim == 128) launch_store_for<128>(p, grid, block, mode, stream);
  else launch_store_for<64>(p, grid, block, mode, stream);
  return hipGetLastError();
}

hipError_t launch_load_kv(const LoadParams& p, int64_t n_units, int head_dim, int32_t kv_dtype, hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  const HeadGrid kv = head_grid(p.num_kv_heads, head_dim, false);
  const dim3 grid((unsigned)n_units, kv.groups), block(kv.threads);
  if (head_dim == 128) launch_load_for<128>(p, grid, block, kv_dtype, stream);
  else launch_load_for<64>(p, grid, block, kv_dtype, stream);
  return hipGetLastError();
}

}  // namespace kvx
