// Attention of (suffix token, head) rows to the latent cache entries themselves, gfx950.
#include <type_traits>

#include "kvx_latent_tile.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;

// A tile of 64 keys in LDS: pages of 16 rows, in a page its two halves of 8 rows, in a half
// blocks of 128 bytes of the rows: [page][half][block][8 rows][128 bytes], where a wave-wide
// direct load of 1 KiB fills one block from one lane offset.  The eight 16-byte chunks of a
// row in a block are stored in the order c ^ swz(row): rows are 32 banks apart modulo 64,
// and this moves the rows of an operand read (16 rows one chunk; 4 rows two chunks) to
// different banks.
template <int LAT>
struct TileAt {
  static constexpr int HALF = 8 * LatGeom<LAT>::ROWB;
  __device__ static int row(int r) { return (r >> 3) * HALF + (r & 7) * 128; }
  __device__ static int chunk(int r, int c) { return row(r) + (c >> 3) * 1024 + (((c & 7) ^ swz(r)) << 4); }
};

template <int LAT, bool FP8>
struct Loader;

template <int LAT>
struct Loader<LAT, false> {
  using G = LatGeom<LAT>;
  static constexpr int BLOCKS = G::ROWB / 128;
  int off;  // of this lane in a block of the first half; the second half's has bit 4 flipped
  const uint8_t* base;
  const int32_t* ids;
  int64_t page_bytes;
  int key_end, safe, lane, wave;
  uint32_t page;  // of the next tile to load

  __device__ __forceinline__ uint32_t page_at(int k0) const {
    int lp = k0 / kPageSize + wave;
    const int last = (key_end - 1) / kPageSize;
    return (uint32_t)((const_i32_ptr)ids)[lp < last ? lp : last];
  }
  __device__ __forceinline__ void init(const LatentAttnParams& p, const LatentUnit& u, int safe_key, int l, int w) {
    base = p.pool.base;
    ids = p.pool.page_ids + u.page_base;
    page_bytes = p.pool.page_bytes;
    key_end = u.key_end;
    safe = safe_key;
    lane = l;
    wave = w;
    off = (l >> 3) * G::ROWB + (((l & 7) ^ swz(l >> 3)) << 4);
    page = page_at(u.key_begin);
  }
  // Tokens k0 .. k0 + 63; those at or past key_end become token `safe`.
  __device__ __forceinline__ void issue(uint8_t* tile, int k0) {
    const uint32_t lds = lds_address(tile + wave * (16 * G::ROWB));
    if (k0 + kLatTileKeys <= key_end) {
      const uint8_t* src = base + (uint64_t)page * page_bytes;
#pragma unroll
      for (int i = 0; i < BLOCKS; i++) lds_load_1k(src + i * 128, off, lds + i * 1024);
#pragma unroll
      for (int i = 0; i < BLOCKS; i++)
        lds_load_1k(src + 8 * G::ROWB + i * 128, off ^ 16, lds + (BLOCKS + i) * 1024);
    } else {
      const uint32_t sp = (uint32_t)((const_i32_ptr)ids)[safe / kPageSize];
      const uint8_t* src = base + (uint64_t)page * page_bytes;
      const uint8_t* alt = base + (uint64_t)sp * page_bytes + (safe % kPageSize) * G::ROWB;
      const int left = key_end - k0 - wave * kPageSize;  // rows of this page that exist
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int row = 8 * h + (lane >> 3), c = ((lane & 7) ^ swz(row)) << 4;
        const uint8_t* from = (row < left ? src + row * G::ROWB : alt) + c;
#pragma unroll
        for (int i = 0; i < BLOCKS; i++) lds_load_1k(from + i * 128, lds + (h * BLOCKS + i) * 1024);
      }
    }
    page = page_at(k0 + kLatTileKeys);
  }
  __device__ __forceinline__ void finish(uint8_t*) {}
};

// An 8-bit page comes through registers, 16 codes a lane and load, issued a tile ahead, and
// is written to LDS as bf16 (exactly: code * 2^e) once the products of the tile before are
// done.
template <int LAT>
struct Loader<LAT, true> {
  using G = LatGeom<LAT>;
  static constexpr int LOADS = LAT / 64;       // of codes: 1 KiB each, 1024 / LAT slots
  static constexpr int LPS = LAT / 16;         // lanes per slot
  static constexpr int SPL = 64 / LPS;         // slots per load
  const uint8_t* base;
  const int32_t* ids;
  int64_t page_bytes;
  int key_end, safe, lane, wave;
  uint32_t page;
  uint4 codes[LOADS];
  uint4 key[2];
  uint64_t scales;  // LOADS bytes, one per load

  __device__ __forceinline__ uint32_t page_at(int at) const {
    int lp = at / kPageSize + wave;
    const int last = (key_end - 1) / kPageSize;
    return (uint32_t)((const_i32_ptr)ids)[lp < last ? lp : last];
  }
  __device__ __forceinline__ void init(const LatentAttnParams& p, const LatentUnit& u, int safe_key, int l, int w) {
    base = p.pool.base;
    ids = p.pool.page_ids + u.page_base;
    page_bytes = p.pool.page_bytes;
    key_end = u.key_end;
    safe = safe_key;
    lane = l;
    wave = w;
    page = page_at(u.key_begin);
  }
  __device__ __forceinline__ void issue(uint8_t*, int k0) {
    const uint8_t* src = base + (uint64_t)page * page_bytes;
    constexpr int SC = kPageSize * (LAT + 2 * kLatRope);
    const int left = key_end - k0 - wave * kPageSize, sub = lane / LPS, grp = (lane % LPS) / 4;
    const uint8_t* sc = src + SC + latent_scale_at(LAT, sub, grp);
    if constexpr (LOADS == 8) scales = *(const uint64_t*)sc;
    else scales = *(const uint32_t*)sc;
    if (left >= kPageSize) {
#pragma unroll
      for (int i = 0; i < LOADS; i++) codes[i] = *(const uint4*)(src + i * 1024 + lane * 16);
#pragma unroll
      for (int i = 0; i < 2; i++) key[i] = *(const uint4*)(src + kPageSize * LAT + i * 1024 + lane * 16);
    } else {  // slots that the request does not own: the safe token's
      const uint8_t* alt = base + (uint64_t)(uint32_t)((const_i32_ptr)ids)[safe / kPageSize] * page_bytes;
      const int ss = safe % kPageSize;
      const uint64_t b = alt[SC + latent_scale_at(LAT, ss, grp)];
#pragma unroll
      for (int i = 0; i < LOADS; i++) {
        const int slot = i * SPL + sub, c = lane % LPS;
        if (slot >= left) scales = (scales & ~(0xFFull << (8 * i))) | b << (8 * i);
        codes[i] = *(const uint4*)((slot < left ? src + slot * LAT : alt + ss * LAT) + c * 16);
      }
#pragma unroll
      for (int i = 0; i < 2; i++) {
        const int slot = i * 8 + lane / 8, c = lane % 8;
        key[i] = *(const uint4*)((slot < left ? src + slot * 128 : alt + ss * 128) + kPageSize * LAT + c * 16);
      }
    }
    page = page_at(k0 + kLatTileKeys);
  }
  __device__ __forceinline__ void finish(uint8_t* tile) {
    uint8_t* rows = tile + wave * (16 * G::ROWB);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const int slot = i * SPL + lane / LPS, c = lane % LPS;
      const float sc = __uint_as_float((uint32_t)(scales >> (8 * i) & 0xFF) << 23);
      const uint32_t w[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
      uint32_t y[8];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        y[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], sc, false));
        y[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], sc, true));
      }
      *(uint4*)(rows + TileAt<LAT>::chunk(slot, 2 * c)) = make_uint4(y[0], y[1], y[2], y[3]);
      *(uint4*)(rows + TileAt<LAT>::chunk(slot, 2 * c + 1)) = make_uint4(y[4], y[5], y[6], y[7]);
    }
#pragma unroll
    for (int i = 0; i < 2; i++) *(uint4*)(rows + TileAt<LAT>::chunk(i * 8 + lane / 8, LAT / 8 + lane % 8)) = key[i];
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
  // a token that every row of the unit sees, where there is one
  const int safe = pos0 < u.key_begin ? u.key_begin : (pos0 < u.key_end ? pos0 : u.key_end - 1);
  Loader<LAT, FP8> loader;
  loader.init(p, u, safe, lane, wave);

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
    for (int ks = 0; ks < G::KS; ks++) {
      qf[rb][ks] = __builtin_bit_cast(bf16x8, src[ks * 4 + g]);
      // operands of the unit's whole life go to the accumulator half of the register file
      if constexpr (RBW * G::KS > 32) keep_in_acc(qf[rb][ks]);
    }
  }
  const int full_end = pos0 + 1 < u.key_end ? pos0 + 1 : u.key_end;  // keys before it are seen by every row

  f32x4 o[RB][G::DB];
  float m[RB];    // reference points (log2 units; -inf: no key seen yet)
  float l[RBW];   // this lane's share of its rows' sums
  const float scale = p.scale_log2;
  // LDS offsets of the operands.  Chunk orders differ from row to row in bits 4 to 6 of an
  // offset only, so a few lane offsets and immediates reach every operand.
  uint32_t kat[2];  // score product: 32 dims a step, even and odd steps
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int r = kw * KBW * 16 + n;
    kat[i] = TileAt<LAT>::row(r) + ((i * 64 + g * 16) ^ (swz(r) << 4));
  }
  uint32_t vat[4];  // value product: dim blocks modulo 4 (the second four keys of a lane have bit 6 flipped)
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int r = 8 * g + n / 4;
    vat[i] = TileAt<LAT>::row(r) + wave * (G::DW / 64 * 1024) + ((i * 32 + (n % 4) / 2 * 16) ^ (swz(r) << 4)) +
             (n % 2) * 8;
  }
  uint32_t pw[KBW], pr_at[2];
#pragma unroll
  for (int kb = 0; kb < KBW; kb++)
    pw[kb] = lds_address(pl) + (rw * RBW * 16 + n) * 128 + (((2 * (kw * KBW + kb) + g / 2) ^ (n & 7)) * 16) + (g & 1) * 8;
#pragma unroll
  for (int i = 0; i < 2; i++) pr_at[i] = lds_address(pl) + n * 128 + (((4 * i + g) ^ (n & 7)) * 16);
#pragma unroll
  for (int i = 0; i < 2; i++) opaque(kat[i]), opaque(pr_at[i]);
#pragma unroll
  for (int i = 0; i < 4; i++) opaque(vat[i]);
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
    loader.page = loader.page_at(u.key_begin);
    loader.issue(tile[0], u.key_begin);
    loader.finish(tile[0]);
    int buf = 0;
    for (int k0 = u.key_begin; k0 < u.key_end; k0 += kLatTileKeys, buf ^= 1) {
      const lds_ptr cur = (lds_ptr)tile[0] + buf * G::TILE;
      uint8_t* nxt = tile[buf ^ 1];
      const bool more = k0 + kLatTileKeys < u.key_end;
      if constexpr (!FP8) wait_vmcnt<0>();
      __syncthreads();  // the tile is whole, and every wave has done with the one before
      if (more) loader.issue(nxt, k0 + kLatTileKeys);

      f32x4 s[RBW][KBW];
#pragma unroll
      for (int rb = 0; rb < RBW; rb++)
#pragma unroll
        for (int kb = 0; kb < KBW; kb++) s[rb][kb] = f32x4{};
      // Operand reads run ahead of their products: a step is 16 RBW cycles of MFMA, a read
      // from LDS takes some 130, and nothing else runs on this SIMD meanwhile.
      bf16x8 ka[AK + 1];
      auto read_k = [&](int j) {  // step j: dims 32 (j / KBW) .., key block j % KBW
        const int ks = j / KBW, kb = j % KBW;
        return read_b128(cur + kat[ks & 1] + (ks >> 1) * 1024 + kb * (16 * G::ROWB));
      };
#pragma unroll
      for (int j = 0; j < AK; j++) ka[j] = read_k(j);
#pragma unroll
      for (int j = 0; j < G::KS * KBW; j++) {
        if (j + AK < G::KS * KBW) ka[(j + AK) % (AK + 1)] = read_k(j + AK);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int rb = 0; rb < RBW; rb++)
          s[rb][j % KBW] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[j % (AK + 1)], qf[rb][j / KBW], s[rb][j % KBW], 0,
                                                                   0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (k0 + kLatTileKeys > full_end) {
#pragma unroll
        for (int kb = 0; kb < KBW; kb++) {
          const int key0 = k0 + (kw * KBW + kb) * 16 + 4 * g;
#pragma unroll
          for (int rb = 0; rb < RBW; rb++)
#pragma unroll
            for (int i = 0; i < 4; i++) s[rb][kb][i] = key0 + i <= limit[rb] ? s[rb][kb][i] : -INFINITY;
        }
      }
      if (!FIXED || k0 == u.key_begin) {  // uniform
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
      }
#pragma unroll
      for (int rb = 0; rb < RBW; rb++) {
        const float mr = RW == 1 ? m[rb] : (rw == 0 ? m[rb] : m[RB - RBW + rb]);
        const float ref = mr == -INFINITY ? 0.0f : mr;
#pragma unroll
        for (int kb = 0; kb < KBW; kb++) {
          float pr[4];
#pragma unroll
          for (int i = 0; i < 4; i++) {
            pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][kb][i], scale, -ref));
            l[rb] += pr[i];
          }
          write_b64(pw[kb] + rb * 2048, pack_bf16(pr[0], pr[1]), pack_bf16(pr[2], pr[3]));
        }
      }
      // step j of the value product: 32 keys (j / DB) of dim block j % DB
      bf16x8 va[AV + 1];
      auto read_v = [&](int j) {
        const int k2 = j / G::DB, db = j % G::DB;
        s16x4 h[2];
#pragma unroll
        for (int e = 0; e < 2; e++)
          h[e] = read_tr(cur + vat[(db & 3) ^ (2 * e)] + k2 * (32 * G::ROWB) + e * 512 + (db >> 2) * 1024);
        return join(h[0], h[1]);
      };
#pragma unroll
      for (int j = 0; j < AV; j++) va[j] = read_v(j);
      __syncthreads();
      bf16x8 pb[2][RB];
      auto read_p = [&](int k2) {
#pragma unroll
        for (int rb = 0; rb < RB; rb++) pb[k2][rb] = read_b128(lds_at(pr_at[k2]) + rb * 2048);
      };
      read_p(0);
#pragma unroll
      for (int j = 0; j < 2 * G::DB; j++) {
        const int k2 = j / G::DB, db = j % G::DB;
        if (j + AV < 2 * G::DB) va[(j + AV) % (AV + 1)] = read_v(j + AV);
        if (j == G::DB / 2) read_p(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int rb = 0; rb < RB; rb++)
          o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[j % (AV + 1)], pb[k2][rb], o[rb][db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (more) loader.finish(nxt);
    }
    __syncthreads();
  };
  // With the fixed reference bf16 weights and float32 sums keep their relative precision for
  // scores far above it, unless an exponential or a sum overflows: then the keys are gone
  // over again with a reference that moves.
  run(std::true_type{});
  float acc = 0.0f;
#pragma unroll
  for (int rb = 0; rb < RBW; rb++) acc += l[rb];
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

// Log-sum-exp combination of a tile's parts.  Workgroup (merge, row block, 16-dim block of
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
