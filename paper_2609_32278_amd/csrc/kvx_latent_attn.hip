// Attention of (suffix token, head) rows to the latent cache entries themselves, gfx950.
//
//   o = sum_j w_j c_j / sum_j w_j,   w_j = exp(scale * q . (c_j, r_j)),
// one pass over the keys with float32 scores, sums and reference points.  All heads of a token
// see the same entries, so rows of any head and suffix token of a request share a tile of keys:
// a row costs 2 (2 latent_dim + 64) operations a key, a key 2 (latent_dim + 64) bytes for all
// rows (latent_dim + 128 and scales, 8-bit).
//
// Rows.  A unit holds 16, 32 or 64 rows, by the most that a request has: few rows are bound by
// HBM, and fewer of them leave registers for more reads ahead; many by the matrix unit and by
// LDS, from which each product's operands come once a wave.  A decode batch of 128 requests on
// 16 heads: 339 us with 16 rows, 5.5 TB/s read (a large copy reads and writes 5.0 in all, a
// library's sum of 4 GiB reads 3.7 to 4.0).  64 rows at latent_dim 512: the products of 64 keys are 2176 cycles of the
// matrix unit, measured 3.8k a step (8-bit: 4.8k, with its conversions), 0.9 to 1.2 PFLOP/s by
// how evenly a batch fills the CUs; a large library product reaches 1.2 to 1.3.
//
// Waves.  In the value product each of the 4 waves has a quarter of the latent dims and all rows.
// In the score product it has a quarter of the keys and all rows, or, of 64 rows, half of the
// keys and half of the rows: its queries then fit the register file (288 registers otherwise;
// a quarter of the keys and all rows, half of the reads from LDS but the weights formed apart from
// the products, is as fast on bf16 pools: drafts of 32 requests on 64 heads 176 and 174 us, short
// turns 667 and 675).
//
// Roundings: softmax weights to bf16, the operands the matrix unit takes (half a step, 2^-8, of
// each weight; their sum adds the float32 weights); the result to bf16.
#include <type_traits>

#include "kvx_latent_tile.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;

// A tile of 64 keys in LDS: pages of 16 rows, in a page its two halves of 8 rows, in a half
// blocks of 128 bytes of the rows: [page][half][block][8 rows][128 bytes], where a wave-wide
// direct load of 1 KiB fills one block.  The eight 16-byte chunks of a row in a block are
// stored in the order c ^ order(row).  Score operands are read as chunk 2 g + (0 or 1) of 16
// rows, value operands as two neighbouring chunks of 4 rows; with this order both meet every
// bank once (counted: none of their reads conflict).
template <int LAT>
struct TileAt {
  static constexpr int HALF = 8 * LatGeom<LAT>::ROWB;
  __device__ static int order(int r) { return (r & 2) | ((r >> 1) & 4) | ((r >> 2) & 1); }
  __device__ static int row(int r) { return (r >> 3) * HALF + (r & 7) * 128; }
  __device__ static int chunk(int r, int c) { return row(r) + (c >> 3) * 1024 + (((c & 7) ^ order(r)) << 4); }
};

// How a wave brings its page of a 64-key tile to LDS.  Tokens at or past key_end become the
// last one before it in the page (or, in a page past the last, the last of all).  Loads and
// writes are made one by one among the products of the tile before: a burst of them stalls the
// wave (18 loads of 1 KiB took 1.8k cycles of a step's 5.5k).
template <int LAT>
struct Pages {
  const uint8_t* base;
  const_i32_ptr ids;
  int64_t page_bytes;
  int key_end, lane, wave;
  uint32_t page;       // of the next tile: read at the end of a step, as a scalar load under way
                       // would make every wait for LDS a full drain
  const uint8_t* src;  // the page that is being loaded

  __device__ __forceinline__ uint32_t page_at(int k0) const {
    const int lp = k0 / kPageSize + wave, last = (key_end - 1) / kPageSize;
    return (uint32_t)ids[lp < last ? lp : last];
  }
  __device__ __forceinline__ void init(const LatentAttnParams& p, const LatentUnit& u, int l, int w) {
    base = p.pool.base;
    ids = (const_i32_ptr)(p.pool.page_ids + u.page_base);
    page_bytes = p.pool.page_bytes;
    key_end = u.key_end;
    lane = l;
    wave = w;
  }
  // the page of tile k0, and its last slot that is read
  __device__ __forceinline__ int enter(int k0) {
    src = base + (uint64_t)page * page_bytes;
    const int left = key_end - k0 - wave * kPageSize;
    return left >= kPageSize ? kPageSize - 1 : (left > 0 ? left - 1 : (key_end - 1) % kPageSize);
  }
};

template <int LAT, bool FP8>
struct Loader;

template <int LAT>
struct Loader<LAT, false> : Pages<LAT> {
  using G = LatGeom<LAT>;
  using P = Pages<LAT>;
  static constexpr int BLOCKS = G::ROWB / 128, LOADS = 2 * BLOCKS;
  int from[2];  // of this lane in each half of the page
  uint32_t to;

  __device__ __forceinline__ void begin(uint32_t tile, int k0) {
    const int last = P::enter(k0);
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int row = 8 * h + (P::lane >> 3), c = ((P::lane & 7) ^ TileAt<LAT>::order(row)) << 4;
      from[h] = (row < last ? row : last) * G::ROWB + c;
    }
    to = tile + P::wave * (16 * G::ROWB);
  }
  __device__ __forceinline__ void issue(int i) { lds_load_1k(P::src + i % BLOCKS * 128, from[i / BLOCKS], to + i * 1024); }
};

// An 8-bit page comes through registers, 16 codes a lane and load, and is written to LDS as
// bf16 (exactly: code * 2^e).  Beside the value product of a tile, the next tile's pieces are
// written, each followed by the load of the same piece of the tile after that.
//
// A load takes 8 slots x 128 codes: lanes 8 i .. 8 i + 7 slots i % 4 and i % 4 + 4, whose chunk
// orders differ in bit 0, so that the even (and the odd) chunks that eight lanes write fill
// half a row of banks.
template <int LAT>
struct Loader<LAT, true> : Pages<LAT> {
  using G = LatGeom<LAT>;
  using P = Pages<LAT>;
  static constexpr int CODES = LAT / 64, PER = LAT / 128;  // loads of codes: of a page, of 8 slots
  static constexpr int LOADS = CODES + 2;
  uint32_t from[2];  // codes of this lane's slot in each half
  uint32_t key[2];
  uint4 data[LOADS];
  uint64_t scales, scales_next;  // CODES bytes, one per load
  uint32_t at, key_at;           // this lane's first chunk, and its chunk of the key, in the first half
  uint32_t to;

  __device__ __forceinline__ int sub() const { return ((P::lane >> 3) & 3) | (P::lane & 4); }
  __device__ __forceinline__ void init(const LatentAttnParams& p, const LatentUnit& u, int l, int w) {
    P::init(p, u, l, w);
    at = w * (16 * G::ROWB) + TileAt<LAT>::chunk(sub(), 2 * (l & 3)) + (l >> 5) * 1024;
    key_at = w * (16 * G::ROWB) + TileAt<LAT>::chunk(l >> 3, LAT / 8 + (l & 7));
  }
  __device__ __forceinline__ void begin(uint32_t tile, int k0) {  // `tile` is where finish() writes meanwhile
    constexpr int SC = kPageSize * (LAT + 2 * kLatRope);
    const int last = P::enter(k0);
    const int c = (P::lane >> 5) * 4 + (P::lane & 3);
    const uint8_t* sc = P::src + (uint32_t)(SC + latent_scale_at(LAT, sub(), P::lane >> 5));
    if constexpr (CODES == 8) scales_next = *(const uint64_t*)sc;
    else scales_next = *(const uint32_t*)sc;
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int slot = 8 * h + sub(), ks = 8 * h + (P::lane >> 3);
      from[h] = (slot < last ? slot : last) * LAT + c * 16;
      key[h] = kPageSize * LAT + (ks < last ? ks : last) * 128 + (P::lane & 7) * 16;
    }
    if (last < kPageSize - 1) {  // uniform
#pragma unroll
      for (int i = 0; i < CODES; i++)
        if (8 * (i / PER) + sub() > last)
          scales_next = (scales_next & ~(0xFFull << (8 * i))) |
                        (uint64_t)P::src[SC + latent_scale_at(LAT, last, 2 * (i % PER) + (P::lane >> 5))] << (8 * i);
    }
    to = tile;
  }
  __device__ __forceinline__ void issue(int i) {
    data[i] = *(const uint4*)(P::src + (i < CODES ? from[i / PER] + i % PER * 128 : key[i - CODES]));
  }
  // A quarter of a piece's conversion, and its writes.
  uint32_t y[4];
  __device__ __forceinline__ void finish(int i, int e) {
    // slots 8 and up: the second half, where bit 2 of the chunk order is flipped
    const uint32_t half = (i < CODES ? i / PER : i - CODES) ? TileAt<LAT>::HALF : 0, flip = half ? 64 : 0;
    if (i < CODES) {
      const float sc = __uint_as_float(((uint32_t)(scales >> (8 * i)) & 0xFF) << 23);
      const uint32_t w = e == 0 ? data[i].x : (e == 1 ? data[i].y : (e == 2 ? data[i].z : data[i].w));
      y[2 * e % 4] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, false));
      y[2 * e % 4 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, true));
      formed(y[2 * e % 4]);
      formed(y[2 * e % 4 + 1]);
      if (e % 2) write_b128((at ^ flip ^ (e == 3 ? 16 : 0)) + to + half + i % PER * 2048, y[0], y[1], y[2], y[3]);
    } else if (e == 0) {
      write_b128((key_at ^ flip) + to + half, data[i].x, data[i].y, data[i].z, data[i].w);
    }
  }
};

// Where the units are: in memory, or in the arguments that follow the parameters.
struct InMemory {};

__device__ __forceinline__ LatentUnit unit_of(const LatentAttnParams& p, const InMemory&) { return p.units[blockIdx.x]; }
__device__ __forceinline__ LatentUnit unit_of(const LatentAttnParams&, const LatentSmallPlan& plan) {
  const uint32_t code = plan.code[blockIdx.x];
  LatentUnit u{};
  if (code == kLatNoUnit) return u;
  const LatentSmallTile& t = plan.tile[code >> 10];
  const int c = code & (kLatSmallParts - 1);
  u.row0 = t.row0;
  u.nrows = t.nrows;
  u.qo = t.qo;
  u.prefix = t.prefix;
  u.page_base = t.page_base;
  u.key_begin = c * t.len;
  u.key_end = t.key_end < u.key_begin + t.len ? t.key_end : u.key_begin + t.len;
  u.part = t.key_end > t.len ? t.part0 + c : -1;
  return u;
}
__device__ __forceinline__ LatentUnit unit_of(const LatentAttnParams& p, const LatentRowPlan& plan) {
  const int lane = threadIdx.x & 63, b = (int)blockIdx.x;
  static_assert(kLatRowReqs == 128, "two requests a lane");
  const int r = __popcll(__ballot(plan.first[lane] <= b)) + __popcll(__ballot(plan.first[64 + lane] <= b)) - 1;
  LatentUnit u;
  const int len = plan.len[r], c = b - plan.first[r], end = plan.prefix[r] + plan.extend[r];
  u.row0 = 0;
  u.nrows = plan.extend[r] * p.num_q_heads;
  u.qo = plan.qo[r];
  u.prefix = plan.prefix[r];
  u.page_base = plan.page_base[r];
  u.key_begin = c * len;
  u.key_end = end < u.key_begin + len ? end : u.key_begin + len;
  u.part = end > len ? plan.part0[r] + c : -1;
  return u;
}
__device__ __forceinline__ LatentMerge merge_of(const LatentMergeParams& p, const LatentRowPlan& plan) {
  const int r = blockIdx.x, len = plan.len[r], end = plan.prefix[r] + plan.extend[r];
  return {0, plan.extend[r] * p.num_q_heads, plan.qo[r], plan.part0[r], end > len ? (end + len - 1) / len : 0, 0};
}
__device__ __forceinline__ LatentMerge merge_of(const LatentMergeParams& p, const InMemory&) {
  return p.merges[blockIdx.x];
}
__device__ __forceinline__ LatentMerge merge_of(const LatentMergeParams&, const LatentSmallPlan& plan) {
  const LatentSmallTile& t = plan.tile[blockIdx.x];
  return {t.row0, t.nrows, t.qo, t.part0, t.key_end > t.len ? (t.key_end + t.len - 1) / t.len : 0, 0};
}

template <int LAT, bool FP8, int RB, class Plan>
__global__ __launch_bounds__(kThreads, 1) void latent_attn_kernel(LatentAttnParams p, Plan plan) {
  using G = LatGeom<LAT>;
  constexpr int RW = RB == 4 ? 2 : 1, KW = 4 / RW;  // waves by rows and by keys in the score product
  constexpr int RBW = RB / RW, KBW = 4 / KW;        // 16-row and 16-key blocks of a wave in it
  constexpr int QS = G::KS * KBW;                   // its steps
  // Direct loads of the next tile, as positions in score steps (half value steps from QS on): over
  // the score product and, of 64 rows, a quarter of the value product (drafts of 32 requests on 64
  // heads 182 us over three quarters of the scores, 178 over the scores, 174 so), or, of 16 rows,
  // where HBM and not the matrix unit is the bound, all at its start (4 requests on 16 heads 18.7 us,
  // spread 19.0; 128 requests 339 either way).
  constexpr int SPAN = RB == 1 ? 0 : (RB == 4 ? QS * 11 / 9 : QS);
  // operand reads ahead of their products, in steps of the score and of the value product
  constexpr int AK = RBW == 1 ? 8 : 6, AV = RB == 1 ? 8 : (RB == 2 ? 5 : 3);
  __shared__ __attribute__((aligned(1024))) uint8_t tile[2][G::TILE];
  __shared__ __attribute__((aligned(16))) uint8_t pl[RB * 16 * 128];  // softmax weights [row][key]
  float (*red)[RB * 16] = (float (*)[RB * 16])pl;  // between the waves, while no weights are there
  static_assert(sizeof pl >= 5 * RB * 16 * sizeof(float), "the waves' values fit");
  const LatentUnit u = unit_of(p, plan);
  if (u.nrows == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int kw = wave % KW, rw = wave / KW;
  const int Hq = p.num_q_heads;
  const int64_t flat0 = (int64_t)u.qo * Hq + u.row0;

  const int pos0 = u.prefix + u.row0 / Hq;
  using L = Loader<LAT, FP8>;
  L loader;
  loader.init(p, u, lane, wave);
  const uint32_t tile0 = lds_address(tile);
  auto first_loads = [&]() {
    loader.page = loader.page_at(u.key_begin);
    loader.begin(tile0, u.key_begin);
#pragma unroll
    for (int i = 0; i < L::LOADS; i++) loader.issue(i);
  };
  first_loads();  // ahead of the queries', which then arrive with them

  bf16x8 qf[RBW][G::KS];
  int limit[RBW];  // last visible key of the lane's rows
#pragma unroll
  for (int rb = 0; rb < RBW; rb++) {
    const int row = (rw * RBW + rb) * 16 + n;
    const bool valid = row < u.nrows;
    const int pos = u.prefix + (u.row0 + (valid ? row : 0)) / Hq;
    limit[rb] = pos < u.key_end ? pos : u.key_end - 1;
    const uint4* src = (const uint4*)(p.q + (flat0 + (valid ? row : 0)) * G::ROW);
#pragma unroll
    for (int ks = 0; ks < G::KS; ks++) {  // step ks, lanes g: chunk 2 g + ks % 2 of the step pair's eight
      qf[rb][ks] = __builtin_bit_cast(bf16x8, src[(ks >> 1) * 8 + 2 * g + (ks & 1)]);
      // operands of the unit's whole life go to the accumulator half of the register file
      if constexpr (RBW * G::KS > 32) keep_in_acc(qf[rb][ks]);
    }
  }
  const int full_end = pos0 + 1 < u.key_end ? pos0 + 1 : u.key_end;  // keys before it are seen by every row

  f32x4 o[RB][G::DB];
  float m[RB];    // reference points (log2 units; -inf: no key seen yet)
  float l[RBW];   // this lane's share of its rows' sums
  float neg[RBW]; // its rows' reference points, negated; 0 where there is none
  const float scale = p.scale_log2;
  // LDS offsets of the operands.  Chunk orders differ from row to row in bits 4 to 6 of an
  // offset only, so a few lane offsets and immediates reach every operand.
  uint32_t kat[2];  // score product: 32 dims a step, even and odd steps
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int r = kw * 16 + n;
    kat[i] = TileAt<LAT>::chunk(r, 2 * g + i);
  }
  uint32_t vat[2][4];  // value product: first and second four keys of a lane, dim blocks modulo 4
#pragma unroll
  for (int e = 0; e < 2; e++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      vat[e][i] = TileAt<LAT>::chunk(8 * g + 4 * e + n / 4, 2 * i + (n % 4) / 2) + wave * (G::DW / 64 * 1024) + (n % 2) * 8;
      opaque(vat[e][i]);
    }
  uint32_t pw[KBW], pr_at[2];
#pragma unroll
  for (int kb = 0; kb < KBW; kb++)
    pw[kb] = lds_address(pl) + (rw * RBW * 16 + n) * 128 + (((2 * (kb * KW + kw) + g / 2) ^ (n & 7)) * 16) + (g & 1) * 8;
#pragma unroll
  for (int i = 0; i < 2; i++) pr_at[i] = lds_address(pl) + n * 128 + (((4 * i + g) ^ (n & 7)) * 16);
#pragma unroll
  for (int i = 0; i < 2; i++) opaque(kat[i]), opaque(pr_at[i]);
#pragma unroll
  for (int kb = 0; kb < KBW; kb++) opaque(pw[kb]);

  // One pass over the keys.  FIXED: the reference point stays at the first tile's row maximum.
  auto run = [&](auto fixed) {
    constexpr bool FIXED = decltype(fixed)::value;
#pragma unroll
    for (int rb = 0; rb < RBW; rb++) l[rb] = 0.0f;
#pragma unroll
    for (int rb = 0; rb < RB; rb++) {
      m[rb] = -INFINITY;
#pragma unroll
      for (int db = 0; db < G::DB; db++) o[rb][db] = f32x4{};
    }
    if constexpr (!FIXED) first_loads();
    if constexpr (FP8) {
      loader.page = loader.page_at(u.key_begin + kLatTileKeys);
      loader.scales = loader.scales_next;
#pragma unroll
      for (int i = 0; i < L::LOADS; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) loader.finish(i, e);
      loader.begin(tile0, u.key_begin + kLatTileKeys);
#pragma unroll
      for (int i = 0; i < L::LOADS; i++) loader.issue(i);
    }
    loader.page = loader.page_at(u.key_begin + (FP8 ? 2 : 1) * kLatTileKeys);
    int buf = 0;
    for (int k0 = u.key_begin; k0 < u.key_end; k0 += kLatTileKeys, buf ^= 1) {
      const lds_ptr cur = (lds_ptr)tile[0] + buf * G::TILE;
      if constexpr (!FP8) wait_vmcnt<0>();
      __syncthreads();  // the tile is whole, and every wave has done with the one before

      f32x4 s[RBW][KBW];
      // Operand reads run ahead of their products: a step is 16 RBW cycles of MFMA, a read
      // from LDS takes some 130, and nothing else runs on this SIMD meanwhile.
      bf16x8 ka[AK + 1];
      auto read_k = [&](int j) {  // step j: key block j / KS, dims 32 (j % KS) ..
        const int ks = j % G::KS, kb = j / G::KS;
        return read_b128(cur + kat[ks & 1] + (ks >> 1) * 1024 + kb * (KW * 16 * G::ROWB));
      };
      // Scores of the tile; between(j) runs beside the products of step j.
      auto scores = [&](auto between) {
#pragma unroll
        for (int rb = 0; rb < RBW; rb++)
#pragma unroll
          for (int kb = 0; kb < KBW; kb++) s[rb][kb] = f32x4{};
#pragma unroll
        for (int j = 0; j < AK; j++) ka[j] = read_k(j);
#pragma unroll
        for (int j = 0; j < QS; j++) {
          if (j + AK < QS) ka[(j + AK) % (AK + 1)] = read_k(j + AK);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int rb = 0; rb < RBW; rb++)
            s[rb][j / G::KS] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[j % (AK + 1)], qf[rb][j % G::KS],
                                                                       s[rb][j / G::KS], 0, 0, 0);
          between(j);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      auto mask = [&](int kb) {
        if (k0 + kLatTileKeys > full_end) {
          const int key0 = k0 + (kb * KW + kw) * 16 + 4 * g;
#pragma unroll
          for (int rb = 0; rb < RBW; rb++)
#pragma unroll
            for (int i = 0; i < 4; i++) s[rb][kb][i] = key0 + i <= limit[rb] ? s[rb][kb][i] : -INFINITY;
        }
      };
      if (!FIXED || k0 == u.key_begin) {  // uniform: the reference points, from scores of their own
        scores([](int) {});
#pragma unroll
        for (int kb = 0; kb < KBW; kb++) mask(kb);
#pragma unroll
        for (int rb = 0; rb < RBW; rb++) {
          float mx = -INFINITY;
#pragma unroll
          for (int kb = 0; kb < KBW; kb++)
            mx = fmaxf(mx, fmaxf(fmaxf(s[rb][kb][0], s[rb][kb][1]), fmaxf(s[rb][kb][2], s[rb][kb][3])));
          mx *= scale;
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          if (g == 0) red[kw][(rw * RBW + rb) * 16 + n] = mx;
        }
        __syncthreads();
#pragma unroll
        for (int rb = 0; rb < RB; rb++) {
          float m_new = m[rb];
#pragma unroll
          for (int k = 0; k < KW; k++) m_new = fmaxf(m_new, red[k][rb * 16 + n]);
          if constexpr (!FIXED) {
            const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[rb] - m_new);
            if (rb / RBW == rw) l[rb % RBW] *= alpha;
#pragma unroll
            for (int db = 0; db < G::DB; db++) o[rb][db] *= alpha;
          }
          m[rb] = m_new;
        }
        __syncthreads();
#pragma unroll
        for (int rb = 0; rb < RBW; rb++) {
          const float mr = RW == 1 ? m[rb] : (rw == 0 ? m[rb] : m[RB - RBW + rb]);
          neg[rb] = mr == -INFINITY ? 0.0f : -mr;
        }
      }
      // the i-th of a lane's four weights of one row block and key block
      auto weigh = [&](int rb, int kb, int i) {
        s[rb][kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][kb][i], scale, neg[rb]));
        l[rb] += s[rb][kb][i];
        formed(l[rb]);
        if (i == 3)
          write_b64(pw[kb] + rb * 2048, pack_bf16(s[rb][kb][0], s[rb][kb][1]), pack_bf16(s[rb][kb][2], s[rb][kb][3]));
      };
      bf16x8 va[AV + 1], pb[RB];
      auto read_v = [&](int j) {  // step j of the value product: 32 keys (j / DB) of dim block j % DB
        const int k2 = j / G::DB, db = j % G::DB;
        s16x4 h[2];
#pragma unroll
        for (int e = 0; e < 2; e++)
          h[e] = read_tr(cur + vat[e][db & 3] + k2 * (32 * G::ROWB) + (db >> 2) * 1024);
        return join(h[0], h[1]);
      };
      auto read_p = [&](int k2) {
#pragma unroll
        for (int rb = 0; rb < RB; rb++) pb[rb] = read_b128(lds_at(pr_at[k2]) + rb * 2048);
      };
      auto values = [&](int k2, auto between) {
#pragma unroll
        for (int jj = 0; jj < G::DB; jj++) {
          const int j = k2 * G::DB + jj;
          if (j + AV < 2 * G::DB) va[(j + AV) % (AV + 1)] = read_v(j + AV);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int rb = 0; rb < RB; rb++) {
            o[rb][jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[j % (AV + 1)], pb[rb], o[rb][jj], 0, 0, 0);
            if (rb == (FP8 ? 0 : RB - 1)) between(jj);
            // a quarter of a piece beside each product (a whole one behind a step's products: 24
            // long requests on 128 heads 461 us, so 445)
            if constexpr (FP8) {
#pragma unroll
              for (int i = 0; i < L::LOADS; i++)
                if (i * (2 * G::DB) / L::LOADS == j) {
#pragma unroll
                  for (int e = rb * 4 / RB; e < (rb + 1) * 4 / RB; e++) loader.finish(i, e);
                  if (rb == RB - 1) loader.issue(i);
                }
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      // A wave with two key blocks forms the weights of the first beside the scores of the
      // second, and those of the second beside the value products of the first 32 keys.
      if constexpr (FP8) loader.scales = loader.scales_next;
      loader.begin(tile0 + (buf ^ 1) * G::TILE, k0 + (FP8 ? 2 : 1) * kLatTileKeys);
      scores([&](int j) {
        if constexpr (!FP8) {
#pragma unroll
          for (int i = 0; i < L::LOADS; i++)
            if (i * SPAN / L::LOADS == j) loader.issue(i);
        }
        if constexpr (KBW == 2) {
          if (j == G::KS) mask(0);
#pragma unroll
          for (int e = 0; e < 4 * RBW; e++)
            if (j == G::KS + 2 + 5 * (e / 4)) weigh(e / 4, 0, e % 4);
        }
      });
      if constexpr (KBW == 1) {
        mask(0);
#pragma unroll
        for (int e = 0; e < 4 * RBW; e++) weigh(e / 4, 0, e % 4);
      }
#pragma unroll
      for (int j = 0; j < AV; j++) va[j] = read_v(j);
      __syncthreads();
      read_p(0);
      if constexpr (KBW == 2) mask(1);
      values(0, [&](int jj) {
        if constexpr (KBW == 2) {
#pragma unroll
          for (int e = 0; e < 4 * RBW; e++)
            if (jj == 1 + 2 * (e / 4)) weigh(e / 4, 1, e % 4);
        }
        if constexpr (!FP8) {
#pragma unroll
          for (int i = 0; i < L::LOADS; i++)
            if (i * SPAN / L::LOADS >= QS && (i * SPAN / L::LOADS - QS) / 2 == jj) loader.issue(i);
        }
      });
      if constexpr (KBW == 2) __syncthreads();
      read_p(1);
      values(1, [](int) {});
      loader.page = loader.page_at(k0 + (FP8 ? 3 : 2) * kLatTileKeys);
    }
    wait_vmcnt<0>();
    __syncthreads();
  };
  // A reference that moves with every tile would cost two more barriers and a rescaling of every
  // sum a tile.  With the fixed reference bf16 weights and float32 sums keep their relative precision for
  // scores far above it, unless an exponential or a sum overflows, or the first tile held no
  // score above -inf for a row that sees some of it: then the keys are gone over again with a
  // reference that moves.
  run(std::true_type{});
  float acc = 0.0f;
#pragma unroll
  for (int rb = 0; rb < RBW; rb++) {
    const float mr = RW == 1 ? m[rb] : (rw == 0 ? m[rb] : m[RB - RBW + rb]);
    acc += mr == -INFINITY && limit[rb] >= u.key_begin ? INFINITY : l[rb];
  }
#pragma unroll
  for (int rb = 0; rb < RB; rb++)
#pragma unroll
    for (int db = 0; db < G::DB; db++)
#pragma unroll
      for (int i = 0; i < 4; i++) acc += o[rb][db][i];
  const bool bad = __any(!__builtin_isfinite(acc));
  if (lane == 0) red[wave][0] = bad ? 1.0f : 0.0f;
  __syncthreads();
  const bool again = (red[0][0] + red[1][0]) + (red[2][0] + red[3][0]) > 0.0f;
  __syncthreads();
  if (again) run(std::false_type{});

#pragma unroll
  for (int rb = 0; rb < RBW; rb++) {
    float lt = l[rb];
    lt += __shfl_xor(lt, 16, 64);
    lt += __shfl_xor(lt, 32, 64);
    if (g == 0) red[kw][(rw * RBW + rb) * 16 + n] = lt;
  }
  __syncthreads();
#pragma unroll
  for (int rb = 0; rb < RB; rb++) {
    const int r = rb * 16 + n;
    float lt = red[0][r];
#pragma unroll
    for (int k = 1; k < KW; k++) lt += red[k][r];
    if (m[rb] == INFINITY) lt = NAN;  // inf - inf; the weights against such a reference are 0
    const float inv = lt > 0.0f ? 1.0f / lt : (lt == 0.0f ? 0.0f : lt);
    const float lse2 = lt == 0.0f ? -INFINITY : m[rb] + __log2f(lt);
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

// Log-sum-exp combination of a tile's parts, sums already divided by their totals: latency-bound
// (5 to 17 us).  Workgroup (merge, row block, 16-dim block of
// the latent): 64 lanes hold its 4 sums of 16 rows each; the four waves take every fourth
// part, eight of them in flight, and add up through LDS.
template <int LAT, int RB, class Plan>
__global__ __launch_bounds__(kThreads) void latent_merge_kernel(LatentMergeParams p, Plan plan) {
  using G = LatGeom<LAT>;
  const LatentMerge m = merge_of(p, plan);
  const int rb = blockIdx.y, share = blockIdx.z / G::DB, db = blockIdx.z % G::DB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
  __shared__ f32x4 sums[4][64];
  __shared__ float totals[4][16], tops[16][16];
  if (m.nparts == 0 || rb * 16 >= m.nrows) return;
  const int r = rb * 16 + n;
  const float* lse = p.lse_part + (size_t)m.part0 * (RB * 16) + r;
  float top = -INFINITY;
  for (int i = tid >> 4; i < m.nparts; i += 16) top = fmaxf(top, lse[(size_t)i * (RB * 16)]);
  tops[tid >> 4][n] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; i++) top = fmaxf(top, tops[i][n]);
  const float ref = top == -INFINITY ? 0.0f : top;
  f32x4 o{};
  float total = 0.0f;
  const float* src = p.o_part + (size_t)m.part0 * (RB * 16 * LAT) + (size_t)((share * RB + rb) * G::DB + db) * 256 + lane * 4;
#pragma unroll 8
  for (int i = wave; i < m.nparts; i += 4) {
    const float w = __builtin_amdgcn_exp2f(lse[(size_t)i * (RB * 16)] - ref);
    total += w;
    o += *(const f32x4*)(src + (size_t)i * (RB * 16 * LAT)) * w;
  }
  sums[wave][lane] = o;
  if (g == 0) totals[wave][n] = total;
  __syncthreads();
  if (wave != 0 || r >= m.nrows) return;
  const f32x4 s = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
  total = (totals[0][n] + totals[1][n]) + (totals[2][n] + totals[3][n]);
  const float inv = total > 0.0f ? 1.0f / total : (total == 0.0f ? 0.0f : total);
  const int64_t flat = (int64_t)m.qo * p.num_q_heads + m.row0 + r;
  uint2 w;
  w.x = pack_bf16(s[0] * inv, s[1] * inv);
  w.y = pack_bf16(s[2] * inv, s[3] * inv);
  *(uint2*)(p.out + flat * LAT + share * G::DW + db * 16 + 4 * g) = w;
  if (p.lse != nullptr && blockIdx.z == 0 && g == 0) p.lse[flat] = (ref + __log2f(total)) * kLn2;
}

template <int LAT, bool FP8, class Plan>
void attn_by_blocks(const LatentAttnParams& p, unsigned n, const Plan& plan, int rb, hipStream_t s) {
  if (rb == 1) hipLaunchKernelGGL((latent_attn_kernel<LAT, FP8, 1, Plan>), dim3(n), dim3(kThreads), 0, s, p, plan);
  else if (rb == 2) hipLaunchKernelGGL((latent_attn_kernel<LAT, FP8, 2, Plan>), dim3(n), dim3(kThreads), 0, s, p, plan);
  else hipLaunchKernelGGL((latent_attn_kernel<LAT, FP8, 4, Plan>), dim3(n), dim3(kThreads), 0, s, p, plan);
}

template <class Plan>
void attn_by_pool(const LatentAttnParams& p, unsigned n, const Plan& plan, int latent_dim, bool fp8, int rb,
                  hipStream_t s) {
  if (latent_dim == 512) {
    if (fp8) attn_by_blocks<512, true>(p, n, plan, rb, s);
    else attn_by_blocks<512, false>(p, n, plan, rb, s);
  } else {
    if (fp8) attn_by_blocks<256, true>(p, n, plan, rb, s);
    else attn_by_blocks<256, false>(p, n, plan, rb, s);
  }
}

template <int LAT, class Plan>
void merge_by_blocks(const LatentMergeParams& p, unsigned n, const Plan& plan, int rb, hipStream_t s) {
  const dim3 grid(n, rb, 4 * LatGeom<LAT>::DB), block(kThreads);
  if (rb == 1) hipLaunchKernelGGL((latent_merge_kernel<LAT, 1, Plan>), grid, block, 0, s, p, plan);
  else if (rb == 2) hipLaunchKernelGGL((latent_merge_kernel<LAT, 2, Plan>), grid, block, 0, s, p, plan);
  else hipLaunchKernelGGL((latent_merge_kernel<LAT, 4, Plan>), grid, block, 0, s, p, plan);
}

}  // namespace

hipError_t launch_latent_attention(const LatentAttnParams& p, int64_t n_units, const LatentSmallPlan* small,
                                   const LatentRowPlan* rows, int latent_dim, bool fp8, int row_blocks,
                                   hipStream_t stream) {
  if (rows != nullptr) {
    attn_by_pool(p, (unsigned)rows->n_units, *rows, latent_dim, fp8, row_blocks, stream);
  } else if (small != nullptr) {
    attn_by_pool(p, (unsigned)small->n_units, *small, latent_dim, fp8, row_blocks, stream);
  } else {
    if (n_units <= 0) return hipSuccess;
    attn_by_pool(p, (unsigned)n_units, InMemory{}, latent_dim, fp8, row_blocks, stream);
  }
  return hipGetLastError();
}

hipError_t launch_latent_merge(const LatentMergeParams& p, int64_t n_merges, const LatentSmallPlan* small,
                               const LatentRowPlan* rows, int latent_dim, int row_blocks, hipStream_t stream) {
  if (rows != nullptr) {
    if (latent_dim == 512) merge_by_blocks<512>(p, (unsigned)rows->n, *rows, row_blocks, stream);
    else merge_by_blocks<256>(p, (unsigned)rows->n, *rows, row_blocks, stream);
  } else if (small != nullptr) {
    if (latent_dim == 512) merge_by_blocks<512>(p, (unsigned)small->n_tiles, *small, row_blocks, stream);
    else merge_by_blocks<256>(p, (unsigned)small->n_tiles, *small, row_blocks, stream);
  } else {
    if (n_merges <= 0) return hipSuccess;
    if (latent_dim == 512) merge_by_blocks<512>(p, (unsigned)n_merges, InMemory{}, row_blocks, stream);
    else merge_by_blocks<256>(p, (unsigned)n_merges, InMemory{}, row_blocks, stream);
  }
  return hipGetLastError();
}

}  // namespace kvx
