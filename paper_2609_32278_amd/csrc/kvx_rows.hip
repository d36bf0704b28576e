// Attention of few query rows over all keys of their request, gfx950 (CDNA4): decode steps and
// drafted tokens on a page-scaled pool, and cross attention of few rows (tokens x query heads of one KV
// head) on any pool.
//
// HBM bound: every K and V byte is read once for all rows.  A workgroup of four waves takes one
// KV head of one request over a range of its keys; wave w streams steps w, w + 4, ... of 64 keys
// (32 of a bf16 pool) from the pages straight into registers and multiplies
// them with all rows, in NB blocks of 16:
//   * S^T (keys x rows) = K Q^T on v_mfma_f32_16x16x32_bf16, keys as A straight from memory;
//   * a softmax in base 2 with a running maximum per row, which four lanes share;
//   * O^T += V^T P^T, the 32 keys of a product being those whose weights the lane holds.
// 8-bit codes are converted once for all blocks, with their page's power of two on a page-scaled
// pool.  The registers of a step are refilled with the wave's next one as soon as the products
// have read them.  The waves' results meet in LDS, 16 rows at a time; ranges of a split key range
// by log-sum-exp in a second kernel.
//
// Kernel times: 24 agents of 16k to 131k tokens, 64/8/128 heads, page-scaled pool, 454 us
// (6.3 TB/s); 48 single queries on 200 to 1500 tokens, 16/16/64 heads, bf16 pool, 21.3 us
// (5.4 TB/s); drafts of 1 to 5 tokens of 33 requests on 2k to 20k, 64/8/128 heads, page-scaled pool,
// 112 us and the merge 5.  Each against what was measured in its place: 64 rows a unit (a
// wave then has no registers for loads in flight) 160 us for those drafts against 120; 64 keys a step
// of a bf16 pool 33 us for the single queries against 21; page ids read with the loads that need
// them, not a step ahead, 31 against 21.

#include <type_traits>

#include "kvx_decode_unit.h"

namespace kvx {
namespace {

using decode::bf16x2;
using decode::bf16x8;
using decode::const_i32_ptr;
using decode::f32x4;
using decode::fp8x8_bf16;
using decode::group_max;
using decode::group_sum;
using decode::kLn2;
using decode::load16;
using decode::load8;
using decode::pack2;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

struct RowsUnit {
  int qo_row, ntok, page_base, keys, key_begin, key_end, head, part;
};

__device__ __forceinline__ const_i32_ptr words_of(const RowsParams& p) {
  if (p.words != nullptr) return (const_i32_ptr)p.words;
  return (const_i32_ptr)((const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr() +
                         offsetof(RowsParams, in_args));
}

// The unit of this workgroup: KV heads side by side (scalar loads, uniform).
__device__ __forceinline__ RowsUnit unit_of(const RowsParams& p) {
  const const_i32_ptr w = words_of(p);
  const int i = blockIdx.x / p.num_kv_heads;
  const uint32_t code = (uint32_t)w[kRowsEntryWords * p.n_entries + i];
  const const_i32_ptr e = w + kRowsEntryWords * (code >> kRowsRangeBits);
  const int range = (int)(code & ((1u << kRowsRangeBits) - 1)), len = e[5];
  RowsUnit u;
  u.head = (int)blockIdx.x - i * p.num_kv_heads;
  u.qo_row = e[0];
  u.ntok = e[1];
  u.page_base = e[2];
  u.keys = e[3];
  u.key_begin = range * len;
  u.key_end = u.keys - u.key_begin < len ? u.keys : u.key_begin + len;
  u.part = e[4] < 0 ? -1 : e[4] + u.head * ((u.keys - 1) / len + 1) + range;
  return u;
}

// Whether another request's page list holds this range's first page at the same place (prefixes
// and encodings are shared in whole pages from the start).  Uniform.
__device__ __forceinline__ bool range_is_shared(const RowsParams& p, const RowsUnit& u) {
  const uint32_t* w = p.words;
  if (w == nullptr)
    w = (const uint32_t*)((const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr() +
                          offsetof(RowsParams, in_args));
  const int lp = u.key_begin / kPageSize, own = ((const_i32_ptr)p.page_ids)[u.page_base + lp];
  bool same = false;
  for (int i = threadIdx.x & 63; i < p.n_entries; i += 64) {
    const int base = (int)w[kRowsEntryWords * i + 2], keys = (int)w[kRowsEntryWords * i + 3];
    if (base != u.page_base && lp * kPageSize < keys) same |= p.page_ids[base + lp] == own;
  }
  return __any(same);
}

// Row `row` of a unit's queries among all of them.
__device__ __forceinline__ size_t query_row(const RowsParams& p, const RowsUnit& u, int row) {
  const int tok = row / p.group;
  return (size_t)(u.qo_row + tok) * p.num_q_heads + u.head * p.group + (row - tok * p.group);
}

// Keys that row `row` sees.
__device__ __forceinline__ int row_limit(const RowsParams& p, const RowsUnit& u, int row) {
  return p.causal ? u.keys - (u.ntok - 1 - row / p.group) : u.keys;
}

struct Combine {
  float* o;  // [kWaves][16][D]
  float* m;  // [kWaves][16]
  float* l;
};

// Softmax state of a lane's rows: one of each block.
template <int D, int NB>
struct State {
  f32x4 o[NB][D / 16];
  float m[NB], l[NB];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int b = 0; b < NB; b++) {
#pragma unroll
      for (int i = 0; i < D / 16; i++) o[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[b] = -INFINITY;
      l[b] = 0.f;
    }
  }
  // A step's scores of block b, N fours of keys: their weights as bf16 pairs, and the state moved on.
  template <int N>
  __device__ __forceinline__ void weights(int b, const f32x4 (&s)[N], float scale, uint32_t (&w)[2 * N]) {
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; j++)
#pragma unroll
      for (int i = 0; i < 4; i++) mx = fmaxf(mx, s[j][i]);
    mx = group_max(mx) * scale;
    if (__any(mx > m[b])) {
      const float m_new = fmaxf(m[b], mx);
      const float alpha = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[b] - m_new);
      l[b] *= alpha;
#pragma unroll
      for (int i = 0; i < D / 16; i++) o[b][i] *= alpha;
      m[b] = m_new;
    }
    // a row whose keys so far are all masked keeps m = -inf: its weights are 0
    const float neg = m[b] == -INFINITY ? 0.f : -m[b];
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int e = 0; e < 2 * N; e++) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e / 2][2 * (e % 2)], scale, neg));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e / 2][2 * (e % 2) + 1], scale, neg));
      w[e] = pack2(p0, p1);
      l[b] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[e]), ones, l[b], false);
    }
  }
};

// The waves' results to the unit's: lane (n, g) holds dims 16 i + 4 g .. +3 of row 16 b + n.
// A row without a score above -inf gives zeros and -inf, one whose sum is a NaN gives NaN.
template <int D, int NB>
__device__ __forceinline__ void finish(const RowsParams& p, const RowsUnit& u, Combine sm, const State<D, NB>& st,
                                       float vscale, int part_rows) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, g = lane >> 4, rows = u.ntok * p.group;
#pragma unroll
  for (int b = 0; b < NB; b++) {
    if (16 * b >= rows) break;  // uniform
    if (b > 0) __syncthreads();
    const float l_row = group_sum(st.l[b]);
    if (g == 0) {
      sm.m[wave * 16 + n] = st.m[b];
      sm.l[wave * 16 + n] = l_row;
    }
#pragma unroll
    for (int i = 0; i < D / 16; i++) *(f32x4*)&sm.o[(wave * 16 + n) * D + 16 * i + 4 * g] = st.o[b][i];
    __syncthreads();
    const int live = rows - 16 * b < 16 ? rows - 16 * b : 16;
    for (int idx = threadIdx.x; idx < live * (D / 4); idx += kThreads) {
      const int r = idx / (D / 4), d = 4 * (idx - r * (D / 4)), row = 16 * b + r;
      float M = -INFINITY, e[kWaves];
#pragma unroll
      for (int w = 0; w < kWaves; w++) M = fmaxf(M, sm.m[w * 16 + r]);
      float sum = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; w++) {
        e[w] = sm.m[w * 16 + r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm.m[w * 16 + r] - M);
        sum += e[w] * sm.l[w * 16 + r];
        acc += e[w] * *(const f32x4*)&sm.o[(w * 16 + r) * D + d];
      }
      const float inv = sum > 0.f ? vscale / sum : sum == 0.f ? 0.f : sum;  // NaN stays
      const float lse = sum > 0.f ? (M + __log2f(sum)) * kLn2 : sum == 0.f ? -INFINITY : sum;
      acc *= inv;
      if (u.part < 0) {
        const size_t at = query_row(p, u, row);
        *(uint2*)(p.out + at * D + d) = make_uint2(pack2(acc[0], acc[1]), pack2(acc[2], acc[3]));
        if (p.lse != nullptr && d == 0) p.lse[at] = lse;
      } else {
        const size_t at = (size_t)u.part * part_rows + row;
        *(f32x4*)(p.o_part + at * D + d) = acc;
        if (d == 0) p.lse_part[at] = lse;
      }
    }
  }
}

// ---------------------------------------------------------------- bf16 pool

// A step: a pair of pages.
template <int D>
struct Step16 {
  uint4 k[2][D / 32];  // K A-operands, one per 32-dim step
  uint2 v[2][D / 16];  // V^T: slots 4g .. 4g + 3, one per 16-dim block
};

template <int D, int NB, class Nt>
__device__ __forceinline__ void rows_unit(const RowsParams& p, const RowsUnit& u, Combine sm, Nt&& nt, int part_rows) {
  using S = Step16<D>;
  constexpr int QS = D / 32, DB = D / 16, KEYS = 2 * kPageSize;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  bf16x8 qf[NB][QS];
  int limit[NB];
#pragma unroll
  for (int b = 0; b < NB; b++) {
    const int row = 16 * b + n;
    const bool valid = row < u.ntok * p.group;
    const uint4* src = (const uint4*)(p.q + query_row(p, u, valid ? row : 0) * D + 8 * g);
    limit[b] = valid ? row_limit(p, u, row) : u.keys;
#pragma unroll
    for (int s = 0; s < QS; s++) qf[b][s] = __builtin_bit_cast(bf16x8, valid ? src[4 * s] : make_uint4(0, 0, 0, 0));
  }
  const size_t page_stride = (size_t)p.num_kv_heads * (kPageSize * D), head_off = (size_t)u.head * (kPageSize * D);
  const uint16_t* kbase = (const uint16_t*)p.k_pool + head_off + n * D + 8 * g;
  const uint16_t* vbase = (const uint16_t*)p.v_pool + head_off + n * kPageSize + 4 * g;
  const const_i32_ptr pages = (const_i32_ptr)p.page_ids + u.page_base;
  const int last_page = (u.key_end - 1) / kPageSize, lp0 = u.key_begin / kPageSize;
  const int n_steps = (u.key_end - u.key_begin + KEYS - 1) / KEYS;
  // element offsets of a step's two pages; pages past the end repeat the last one (their keys are
  // masked)
  struct Pages {
    size_t at[2];
  };
  auto pages_of = [&](int step) {
    Pages w;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int l = lp0 + 2 * step + i;
      w.at[i] = (size_t)(uint32_t)pages[l < last_page ? l : last_page] * page_stride;
    }
    return w;
  };
  auto load_k = [&](const Pages& w, S& r, auto nt_flag) {
#pragma unroll
    for (int s = 0; s < QS; s++)
#pragma unroll
      for (int i = 0; i < 2; i++) r.k[i][s] = load16<decltype(nt_flag)::value>(kbase + w.at[i] + 32 * s);
  };
  auto load_v = [&](const Pages& w, S& r, auto nt_flag) {
#pragma unroll
    for (int b = 0; b < DB; b++)
#pragma unroll
      for (int i = 0; i < 2; i++) r.v[i][b] = load8<decltype(nt_flag)::value>(vbase + w.at[i] + 16 * b * kPageSize);
  };
  State<D, NB> st;
  st.clear();
  auto compute = [&](int step, S& r, auto tail_flag, auto nt_flag) {
    constexpr bool TAIL = decltype(tail_flag)::value;
    const int next = step + kWaves;
    const bool more = next < n_steps;  // uniform
    Pages nx{};
    if (more) nx = pages_of(next);
    f32x4 s[NB][2];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
      for (int i = 0; i < 2; i++) s[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < QS; q++)
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int b = 0; b < NB; b++)
          s[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r.k[i][q]), qf[b][q], s[b][i], 0,
                                                            0, 0);
    if (more) load_k(nx, r, nt_flag);
    const int key0 = u.key_begin + KEYS * step + 4 * g;  // of this lane in page i: key0 + 16 i ..
    uint2 va[2][DB];
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int d = 0; d < DB; d++) va[i][d] = r.v[i][d];
    if (more) load_v(nx, r, nt_flag);
    uint32_t w[NB][4];
#pragma unroll
    for (int b = 0; b < NB; b++) {
      if constexpr (TAIL) {
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (key0 + 16 * i + e >= (limit[b] < u.key_end ? limit[b] : u.key_end)) s[b][i][e] = -INFINITY;
      }
      st.weights(b, s[b], p.scale_log2, w[b]);
    }
    if constexpr (TAIL) {  // zero V of keys past the end: unwritten slots may hold NaN
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const int left = u.key_end - (key0 + 16 * i);
        const uint32_t lo = left >= 2 ? 0xFFFFFFFFu : left == 1 ? 0xFFFFu : 0u;
        const uint32_t hi = left >= 4 ? 0xFFFFFFFFu : left == 3 ? 0xFFFFu : 0u;
#pragma unroll
        for (int b = 0; b < DB; b++) {
          va[i][b].x &= lo;
          va[i][b].y &= hi;
        }
      }
    }
#pragma unroll
    for (int d = 0; d < DB; d++) {
      const uint4 a = make_uint4(va[0][d].x, va[0][d].y, va[1][d].x, va[1][d].y);
#pragma unroll
      for (int b = 0; b < NB; b++)
        st.o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, make_uint4(w[b][0], w[b][1], w[b][2], w[b][3])),
            st.o[b][d], 0, 0, 0);
    }
  };
  S r;
  if (wave < n_steps) {
    const Pages w = pages_of(wave);
    load_k(w, r, std::false_type{});
    load_v(w, r, std::false_type{});
  }
  const int all_see = p.causal ? u.keys - (u.ntok - 1) : u.keys;  // keys [0, all_see) are visible to every row
  const int whole = ((all_see < u.key_end ? all_see : u.key_end) - u.key_begin);
  const int n_full = whole > 0 ? whole / KEYS : 0;
  int j = wave;
  if (nt())
    for (; j < n_full; j += kWaves) compute(j, r, std::false_type{}, std::true_type{});
  else
    for (; j < n_full; j += kWaves) compute(j, r, std::false_type{}, std::false_type{});
  for (; j < n_steps; j += kWaves) compute(j, r, std::true_type{}, std::false_type{});
  finish<D, NB>(p, u, sm, st, 1.0f, part_rows);
}

// ---------------------------------------------------------------- 8-bit pools

// A step: four pages.  MFMA j of a k-step holds slots 4j .. 4j+3 of each of them (A row m: slot
// 4j + m % 4 of page m / 4), so that lane group g ends up with page g's scores, whose V is one
// 16-byte load per dim: all 16 slots of the lane's dim of page g.
template <int D>
struct Step8 {
  uint4 k[4][D / 64];
  uint4 v[D / 16];
  float kby, vby;  // page-scaled pool: the powers of two of the lane's K page and V page
};

// 0x80 in every byte of w that is a NaN code
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// NaN codes of c as zeros
__device__ __forceinline__ uint4 without_nans(uint4 c) {
  auto clean = [](uint32_t w) { return w & ~((nan_codes(w) >> 7) * 0xFFu); };
  return make_uint4(clean(c.x), clean(c.y), clean(c.z), clean(c.w));
}

// Rows that see a NaN value get NaN in its dim: where the product of "is NaN" (dims x keys) and "is
// seen" (keys x rows), ones and zeros, is not 0.  v: the lane's codes of the first 16 dims, key0:
// their first slot's key.  Read again, one block after the other: kept for this, or cleaned ahead of
// the products, the codes cost registers (256 for 235 in two blocks of rows, D = 128, or spills).
template <int D, int NB>
__device__ __forceinline__ void nan_to_rows(const char* v, int key0, const int (&limit)[NB], State<D, NB>& st) {
#pragma unroll
  for (int b = 0; b < NB; b++) {
    uint32_t w[8];  // slots 2 e, 2 e + 1: bf16 ones
#pragma unroll
    for (int e = 0; e < 8; e++)
      w[e] = (key0 + 2 * e < limit[b] ? 0x3F80u : 0u) | (key0 + 2 * e + 1 < limit[b] ? 0x3F800000u : 0u);
#pragma unroll
    for (int d = 0; d < D / 16; d++) {
      auto ones = [](uint32_t c) { return (nan_codes(c) >> 7) * 0x38u; };  // e4m3 1.0
      const uint4 c = load16<false>(v + 256 * d);
      f32x4 n = {0.f, 0.f, 0.f, 0.f};
      n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          __builtin_bit_cast(bf16x8, fp8x8_bf16(make_uint2(ones(c.x), ones(c.y)))),
          __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3])), n, 0, 0, 0);
      n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          __builtin_bit_cast(bf16x8, fp8x8_bf16(make_uint2(ones(c.z), ones(c.w)))),
          __builtin_bit_cast(bf16x8, make_uint4(w[4], w[5], w[6], w[7])), n, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; e++) st.o[b][d][e] = n[e] > 0.f ? __builtin_nanf("") : st.o[b][d][e];
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

template <int D, int NB, bool PAGE, class Nt>
__device__ __forceinline__ void rows_unit8(const RowsParams& p, const RowsUnit& u, Combine sm, Nt&& nt, int part_rows) {
  using S = Step8<D>;
  constexpr int KS = D / 64, DB = D / 16, KEYS = 4 * kPageSize;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  bf16x8 qf[NB][KS][2];  // k-step (i, h) takes dims 64 i + 16 g + 8 h .. +8
  int limit[NB];
#pragma unroll
  for (int b = 0; b < NB; b++) {
    const int row = 16 * b + n;
    const bool valid = row < u.ntok * p.group;
    const uint4* src = (const uint4*)(p.q + query_row(p, u, valid ? row : 0) * D + 16 * g);
    limit[b] = valid ? row_limit(p, u, row) : u.keys;
#pragma unroll
    for (int i = 0; i < KS; i++)
#pragma unroll
      for (int h = 0; h < 2; h++)
        qf[b][i][h] = __builtin_bit_cast(bf16x8, valid ? src[8 * i + h] : make_uint4(0, 0, 0, 0));
  }
  const uint32_t page_bytes = (uint32_t)p.num_kv_heads * (kPageSize * D);
  const char* kbase = (const char*)p.k_pool + (size_t)u.head * (kPageSize * D) + (n & 3) * D + 16 * g;
  const char* vbase = (const char*)p.v_pool + (size_t)u.head * (kPageSize * D) + n * kPageSize;
  const const_i32_ptr pages = (const_i32_ptr)p.page_ids + u.page_base;
  const int last_page = (u.key_end - 1) / kPageSize, lp0 = u.key_begin / kPageSize;
  const int n_steps = (u.key_end - u.key_begin + KEYS - 1) / KEYS;
  typedef uint32_t ids_t __attribute__((ext_vector_type(4)));
  auto ids_of = [&](int step) {  // pages past the end repeat the last one (their keys are masked)
    const int l = lp0 + 4 * step;
    auto at = [&](int i) { return (uint32_t)pages[l + i < last_page ? l + i : last_page]; };
    return ids_t{at(0), at(1), at(2), at(3)};
  };
  auto pick = [](const ids_t& w, bool odd, bool high) {
    const uint32_t lo = odd ? w.y : w.x, hi = odd ? w.w : w.z;
    return high ? hi : lo;
  };
  auto scale_at = [&](uint32_t page) { return p.k_scale + 2 * ((uint64_t)page * (uint32_t)p.num_kv_heads + (uint32_t)u.head); };
  auto load_k = [&](const ids_t& w, S& r, auto nt_flag) {
    const uint32_t page = pick(w, n & 4, n & 8);
    const char* src = kbase + (uint64_t)page * page_bytes;
    if constexpr (PAGE) r.kby = scale_at(page)[0];
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
      for (int i = 0; i < KS; i++) r.k[j][i] = load16<decltype(nt_flag)::value>(src + 4 * j * D + 64 * i);
  };
  auto load_v = [&](const ids_t& w, S& r, auto nt_flag) {
    const uint32_t page = pick(w, g & 1, g & 2);
    const char* src = vbase + (uint64_t)page * page_bytes;
    if constexpr (PAGE) r.vby = scale_at(page)[1];
#pragma unroll
    for (int b = 0; b < DB; b++) r.v[b] = load16<decltype(nt_flag)::value>(src + 256 * b);
  };
  const float scale = PAGE ? p.scale_log2 : p.scale_log2 * p.k_scale[u.head];
  const int all_see = p.causal ? u.keys - (u.ntok - 1) : u.keys;  // keys [0, all_see) are visible to every row
  // Some row does not see all of a step's keys: the weight of such a key is 0 there, but 0 * NaN is not.
  // Where NaN came out of a unit with such steps, it is computed again without their NaN codes, and the
  // rows that see these are told.  (Looking at the codes of each such step instead takes 0.5 us of a
  // call on few keys; the look at the sums 0.1 to 0.3.)
  auto hides = [&](int step) {
    const int end = u.key_begin + KEYS * (step + 1);
    return PAGE && (end < u.key_end ? end : u.key_end) > all_see;
  };
  bool again = false;
  State<D, NB> st;
  auto compute = [&](int step, S& r, auto tail_flag, auto nt_flag) {
    constexpr bool TAIL = decltype(tail_flag)::value;
    const int next = step + kWaves;
    const bool more = next < n_steps;  // uniform
    ids_t nx{};
    if (more) nx = ids_of(next);
    f32x4 s[NB][4];
    const float kby = PAGE ? r.kby : 1.0f;
#pragma unroll
    for (int j = 0; j < 4; j++) {
#pragma unroll
      for (int b = 0; b < NB; b++) s[b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KS; i++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const uint4 c = r.k[j][i];
          const bf16x8 a = __builtin_bit_cast(bf16x8, fp8x8_bf16(h ? make_uint2(c.z, c.w) : make_uint2(c.x, c.y), kby));
#pragma unroll
          for (int b = 0; b < NB; b++)
            s[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[b][i][h], s[b][j], 0, 0, 0);
        }
    }
    if (more) load_k(nx, r, nt_flag);
    const int key0 = u.key_begin + KEYS * step + 16 * g;  // slot 0 of the lane group's page
    uint32_t w[NB][8];                                    // weights of slots 2 e, 2 e + 1
#pragma unroll
    for (int b = 0; b < NB; b++) {
      if constexpr (TAIL) {
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (key0 + 4 * j + e >= (limit[b] < u.key_end ? limit[b] : u.key_end)) s[b][j][e] = -INFINITY;
      }
      st.weights(b, s[b], scale, w[b]);
    }
    const float vby = PAGE ? r.vby : 1.0f;
    uint32_t mask[4];  // zeroes V of keys past the end: unwritten slots may hold NaN codes
    if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int left = u.key_end - key0 - 4 * e;  // live slots of this dword
        mask[e] = left >= 4 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
      }
    }
#pragma unroll
    for (int d = 0; d < DB; d++) {
      uint4 c = r.v[d];
      if constexpr (TAIL) c = make_uint4(c.x & mask[0], c.y & mask[1], c.z & mask[2], c.w & mask[3]);
      if (TAIL && PAGE && __builtin_expect(again, 0) && hides(step)) c = without_nans(c);  // uniform
      const bf16x8 lo = __builtin_bit_cast(bf16x8, fp8x8_bf16(make_uint2(c.x, c.y), vby));
      const bf16x8 hi = __builtin_bit_cast(bf16x8, fp8x8_bf16(make_uint2(c.z, c.w), vby));
#pragma unroll
      for (int b = 0; b < NB; b++) {
        st.o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            lo, __builtin_bit_cast(bf16x8, make_uint4(w[b][0], w[b][1], w[b][2], w[b][3])), st.o[b][d], 0, 0, 0);
        st.o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            hi, __builtin_bit_cast(bf16x8, make_uint4(w[b][4], w[b][5], w[b][6], w[b][7])), st.o[b][d], 0, 0, 0);
      }
    }
    if (more) load_v(nx, r, nt_flag);
  };
  const int whole = ((all_see < u.key_end ? all_see : u.key_end) - u.key_begin);
  const int n_full = whole > 0 ? whole / KEYS : 0;
  for (;;) {
    st.clear();
    S r;
    if (wave < n_steps) {
      const ids_t w = ids_of(wave);
      load_k(w, r, std::false_type{});
      load_v(w, r, std::false_type{});
    }
    int j = wave;
    if (nt())
      for (; j < n_full; j += kWaves) compute(j, r, std::false_type{}, std::true_type{});
    else
      for (; j < n_full; j += kWaves) compute(j, r, std::false_type{}, std::false_type{});
    const int first_tail = j;
    for (; j < n_steps; j += kWaves) compute(j, r, std::true_type{}, std::false_type{});
    if (!PAGE || all_see >= u.key_end || first_tail >= n_steps) break;
    if (!again) {
      float sum = 0.f;
#pragma unroll
      for (int b = 0; b < NB; b++)
#pragma unroll
        for (int d = 0; d < DB; d++)
#pragma unroll
          for (int e = 0; e < 4; e++) sum += st.o[b][d][e];
      again = __any(sum != sum);
      if (!again) break;
      continue;
    }
    for (j = first_tail; j < n_steps; j += kWaves)
      if (hides(j)) {
        const char* v = vbase + (uint64_t)pick(ids_of(j), g & 1, g & 2) * page_bytes;
        int seen[NB];
#pragma unroll
        for (int b = 0; b < NB; b++) seen[b] = limit[b] < u.key_end ? limit[b] : u.key_end;
        nan_to_rows<D, NB>(v, u.key_begin + KEYS * j + 16 * g, seen, st);
      }
    break;
  }
  finish<D, NB>(p, u, sm, st, PAGE ? 1.0f : p.v_scale[u.head], part_rows);
}

// NT: see decode_kernel; of more than one block, its second loop spills.  The registers of a
// step in flight allow two waves per SIMD.
template <int D, int KIND, int NB, bool NT>
__global__ __launch_bounds__(kThreads, 2) void rows_kernel(RowsParams p) {
  __shared__ __attribute__((aligned(16))) float o[kWaves * 16 * D];
  __shared__ float m[kWaves * 16], l[kWaves * 16];
  const RowsUnit u = unit_of(p);
  if (u.keys == 0) {  // uniform: nothing to attend to
    for (int64_t i = threadIdx.x; i < (int64_t)u.ntok * p.group * (D / 8); i += kThreads) {
      const int row = (int)(i / (D / 8)), c = (int)(i % (D / 8));
      const size_t at = query_row(p, u, row);
      *(uint4*)(p.out + at * D + 8 * c) = make_uint4(0, 0, 0, 0);
      if (p.lse != nullptr && c == 0) p.lse[at] = -INFINITY;
    }
    return;
  }
  auto nt = [&]() { return NT && !range_is_shared(p, u); };
  if constexpr (KIND == KVX_KV_BF16) rows_unit<D, NB>(p, u, Combine{o, m, l}, nt, 16 * NB);
  else rows_unit8<D, NB, KIND == KVX_KV_FP8_PAGE>(p, u, Combine{o, m, l}, nt, 16 * NB);
}

// Combine the ranges of the entries that have several: o = sum_i e^{lse_i - M} o_i / sum_i e^{lse_i - M}.
// Latency bound: 3 to 5 us and the launch.  (Joined instead by whichever workgroup of an entry ends last, which
// takes a fence of the whole device in every one: 4 agents on 1k to 8k tokens, 32/8/128 heads, 35 us a
// call, 14 so.)  Workgroup (entry, KV head; four rows): D / 4 lanes hold a row's 16-byte columns,
// PG such lane groups take every PG-th range each, and meet in LDS.
constexpr int kMergeRows = 4;
template <int D>
__global__ __launch_bounds__(256) void rows_merge_kernel(RowsParams p) {
  constexpr int C4 = D / 4, PG = 256 / C4 / kMergeRows, UNROLL = 4;
  __shared__ float sm_m[kMergeRows][PG], sm_w[kMergeRows][PG];
  __shared__ f32x4 sm_o[kMergeRows][PG][C4];
  const int i = blockIdx.x / p.num_kv_heads;
  const int c = threadIdx.x % C4, pg = threadIdx.x / C4 % PG, r = threadIdx.x / (C4 * PG);
  const int row = blockIdx.y * kMergeRows + r;
  const const_i32_ptr e = words_of(p) + kRowsEntryWords * i;
  RowsUnit u;
  u.head = (int)blockIdx.x - i * p.num_kv_heads;
  u.qo_row = e[0];
  u.ntok = e[1];
  if (e[4] < 0 || (int)blockIdx.y * kMergeRows >= u.ntok * p.group) return;  // uniform
  const int nparts = (e[3] - 1) / e[5] + 1, part_rows = 16 * p.blocks;
  const int64_t part0 = e[4] + (int64_t)u.head * nparts;
  const bool live = row < u.ntok * p.group;
  const float* lse = p.lse_part + part0 * part_rows + row;
  const float* o = p.o_part + (part0 * part_rows + row) * D + 4 * c;
  float M = -INFINITY, wsum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int q0 = pg; q0 < nparts; q0 += UNROLL * PG) {
    float l[UNROLL];
    f32x4 x[UNROLL];
    float m_new = M;
#pragma unroll
    for (int j = 0; j < UNROLL; j++) {
      const int q = q0 + j * PG;
      const bool in = live && q < nparts;
      l[j] = in ? lse[(size_t)q * part_rows] : -INFINITY;
      x[j] = in ? *(const f32x4*)(o + (size_t)q * part_rows * D) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int j = 0; j < UNROLL; j++) m_new = fmaxf(m_new, l[j]);
    const float alpha = M == -INFINITY ? 0.f : __expf(M - m_new);
    wsum *= alpha;
    acc *= alpha;
#pragma unroll
    for (int j = 0; j < UNROLL; j++) {
      const float w = l[j] == -INFINITY ? 0.f : __expf(l[j] - m_new);  // NaN stays
      wsum += w;
      acc += w * x[j];
    }
    M = m_new;
  }
  sm_o[r][pg][c] = acc;
  if (c == 0) {
    sm_m[r][pg] = M;
    sm_w[r][pg] = wsum;
  }
  __syncthreads();
  if (pg != 0 || !live) return;
#pragma unroll
  for (int j = 1; j < PG; j++) M = fmaxf(M, sm_m[r][j]);
  wsum = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < PG; j++) {
    const float w = sm_m[r][j] == M ? 1.f : __expf(sm_m[r][j] - M);
    wsum += w * sm_w[r][j];
    acc += w * sm_o[r][j][c];
  }
  const float inv = wsum > 0.f ? 1.0f / wsum : wsum == 0.f ? 0.f : wsum;
  const size_t at = query_row(p, u, row);
  *(uint2*)(p.out + at * D + 4 * c) = make_uint2(pack2(acc[0] * inv, acc[1] * inv), pack2(acc[2] * inv, acc[3] * inv));
  if (p.lse != nullptr && c == 0) p.lse[at] = wsum > 0.f ? M + __logf(wsum) : wsum == 0.f ? -INFINITY : wsum;
}

template <int D, int KIND, int NB>
void launch_rows_for(const RowsParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)p.n_codes * (unsigned)p.num_kv_heads), block(kThreads);
  if constexpr (NB == 1) {
    if (p.streams) {
      hipLaunchKernelGGL((rows_kernel<D, KIND, NB, true>), grid, block, 0, stream, p);
      return;
    }
  }
  hipLaunchKernelGGL((rows_kernel<D, KIND, NB, false>), grid, block, 0, stream, p);
}

template <int D, int KIND>
void launch_rows_kind(const RowsParams& p, hipStream_t stream) {
  if (p.blocks == 1) launch_rows_for<D, KIND, 1>(p, stream);
  else launch_rows_for<D, KIND, 2>(p, stream);
}

template <int D>
void launch_rows_dim(const RowsParams& p, hipStream_t stream) {
  if (p.kv_dtype == KVX_KV_BF16) launch_rows_kind<D, KVX_KV_BF16>(p, stream);
  else if (p.kv_dtype == KVX_KV_FP8_E4M3) launch_rows_kind<D, KVX_KV_FP8_E4M3>(p, stream);
  else launch_rows_kind<D, KVX_KV_FP8_PAGE>(p, stream);
  if (!p.any_parts) return;
  const dim3 grid((unsigned)p.n_entries * (unsigned)p.num_kv_heads, (unsigned)(p.rows + kMergeRows - 1) / kMergeRows);
  hipLaunchKernelGGL((rows_merge_kernel<D>), grid, dim3(256), 0, stream, p);
}

}  // namespace

hipError_t launch_rows(const RowsParams& p, int head_dim, hipStream_t stream) {
  if (p.n_codes <= 0) return hipSuccess;
  if (head_dim == 128) launch_rows_dim<128>(p, stream);
  else launch_rows_dim<64>(p, stream);
  return hipGetLastError();
}

}  // namespace kvx
