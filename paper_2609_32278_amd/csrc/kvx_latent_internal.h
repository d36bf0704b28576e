// Declarations shared by the host code and the HIP kernels of latent attention.
#pragma once

#include "kvx_internal.h"
#include "kvx_latent.h"

namespace kvx {

constexpr int kLatRope = 64;        // rope_dim
constexpr int kLatGroup = 64;       // latent values that share a scale on an fp8 pool
constexpr int kLatMinExp = -117;    // their powers of two: every code * 2^e is a finite, normal bf16 value
constexpr int kLatMaxExp = 119;

// Where the scale byte of (slot, group) lies among a page's scale bytes.  A wave that reads a
// page's codes takes 8 slots x 128 codes at once, 16 codes a lane; the bytes that one lane
// meets in these loads lie side by side.
constexpr int latent_scale_at(int latent_dim, int slot, int group) {
  return ((slot % 8) * 2 + group % 2) * (latent_dim / 64) + slot / 8 * (latent_dim / 128) + group / 2;
}

struct LatentPoolView {
  uint8_t* base;
  int64_t page_bytes;
  const int32_t* page_ids;
};

struct LatentStoreParams {
  LatentPoolView pool;
  const uint16_t* kv;
  int64_t kv_stride;        // elements
  const uint16_t* norm;     // bf16 [latent_dim], or null
  float norm_eps;
  int32_t rotate;           // 0: r is copied and there are no queries
  const uint16_t* q;
  uint16_t* q_out;          // may equal q
  int32_t num_q_heads;
  int32_t q_dim;
  int32_t lg_q;             // log2 of the query heads per workgroup (set by the launcher)
  int32_t pad;
  const RopeUnit* units;
  double rev_freq[kLatRope / 2];  // turns per position
  StoreReqs reqs;                 // reqs.n > 0: the units come from here instead
};
static_assert(sizeof(LatentStoreParams) <= 4096, "kernel arguments");

struct LatentLoadParams {
  LatentPoolView pool;
  uint16_t* out;
  int64_t out_stride;
  const RopeUnit* units;
  StoreReqs reqs;
};

hipError_t launch_store_latent(const LatentStoreParams& p, int64_t n_units, int latent_dim, bool fp8, bool interleaved,
                               hipStream_t stream);
hipError_t launch_load_latent(const LatentLoadParams& p, int64_t n_units, int latent_dim, bool fp8,
                              hipStream_t stream);

// ---- attention to the latents themselves

constexpr int kLatTileKeys = 64;     // keys staged in LDS at once; parts start at multiples of it

// One workgroup: rows [row0, row0 + nrows) of a request's (suffix token, head) rows, token
// by token, against keys [key_begin, key_end) of its sequence.
struct LatentUnit {
  int32_t row0;
  int32_t nrows;      // <= 16 * row blocks; 0: padding
  int32_t qo;         // suffix row (of the batch) of the request's first suffix token
  int32_t prefix;     // P
  int32_t page_base;  // offset of the request's page list in page_ids
  int32_t key_begin;  // multiple of kLatTileKeys
  int32_t key_end;    // exclusive
  int32_t part;       // -1: final result; else index of this part's partial result
};
static_assert(sizeof(LatentUnit) == 32, "LatentUnit is 32 bytes");

// A small plan travels in the kernel arguments instead of through a copy: tiles of rows, and
// for each unit in launch order a code word (tile << 10 | part), kLatNoUnit where there is
// none.
constexpr int kLatSmallTiles = 48, kLatSmallUnits = 1024, kLatSmallParts = 1 << 10;
constexpr uint16_t kLatNoUnit = 0xFFFF;
struct LatentSmallTile {
  int32_t row0, nrows, qo, prefix, page_base;
  int32_t key_end;  // keys that a row of the tile sees
  int32_t len;      // keys per part (a multiple of kLatTileKeys)
  int32_t part0;
};
struct LatentSmallPlan {
  int32_t n_units;  // 0: the units are in memory
  int32_t n_tiles;
  LatentSmallTile tile[kLatSmallTiles];
  uint16_t code[kLatSmallUnits];
};

// ... or, where every request is one tile of rows (a decode batch), the requests, longest
// parts first: unit i is part i - first[r] of the last request r with first[r] <= i.
constexpr int kLatRowReqs = 128;
struct LatentRowPlan {
  int32_t n;        // requests
  int32_t n_units;
  int32_t first[kLatRowReqs];  // INT32_MAX past the n-th
  int32_t qo[kLatRowReqs], extend[kLatRowReqs], prefix[kLatRowReqs], page_base[kLatRowReqs];
  int32_t len[kLatRowReqs];    // keys per part
  int32_t part0[kLatRowReqs];
};

// The parts of one tile of rows.
struct LatentMerge {
  int32_t row0, nrows, qo, part0, nparts, pad;
};

struct LatentAttnParams {
  LatentPoolView pool;
  const uint16_t* q;   // bf16 [T, Hq, latent_dim + 64]
  uint16_t* out;       // bf16 [T, Hq, latent_dim]
  float* lse;          // fp32 [T, Hq] or null
  const LatentUnit* units;
  float* o_part;       // fp32 [parts][16 * row blocks * latent_dim], in the accumulators' order
  float* lse_part;     // fp32 [parts][16 * row blocks], base 2
  int32_t num_q_heads;
  float scale_log2;    // sm_scale * log2(e)
};

struct LatentMergeParams {
  const LatentMerge* merges;
  const float* o_part;
  const float* lse_part;
  uint16_t* out;
  float* lse;
  int32_t num_q_heads;
};

static_assert(sizeof(LatentAttnParams) + sizeof(LatentSmallPlan) <= 4096 &&
                  sizeof(LatentAttnParams) + sizeof(LatentRowPlan) <= 4096,
              "kernel arguments");

// small, rows: the plan (in host memory) for the kernel arguments, or null; n_units and
// n_merges are those of a plan in memory.
hipError_t launch_latent_attention(const LatentAttnParams& p, int64_t n_units, const LatentSmallPlan* small,
                                   const LatentRowPlan* rows, int latent_dim, bool fp8, int row_blocks,
                                   hipStream_t stream);
hipError_t launch_latent_merge(const LatentMergeParams& p, int64_t n_merges, const LatentSmallPlan* small,
                               const LatentRowPlan* rows, int latent_dim, int row_blocks, hipStream_t stream);

// ---- per-head weights

// A short list travels in the arguments of the kernel that takes it.
template <typename U, int N>
struct ShortList {
  int32_t n;  // 0: the list is in memory
  U at[N];
};

// A run of suffix tokens of the batch, all heads, and where they are among the tokens that
// take the absorbed form (whose latent-space rows are kept side by side).
struct LatentRows {
  int32_t row0;
  int32_t own0;
  int32_t ntok;  // <= kLatProjTok
  int32_t pad;
};
constexpr int kLatProjTok = 64;
using LatentRowList = ShortList<LatentRows, 64>;

// Per-head products of the absorbed form.  Queries in: [T, Hq, nope + 64] and W_uk to
// [T, Hq, latent + 64].  Sums out: [T, Hq, latent] and W_uv to [T, Hq, v].
struct LatentProjParams {
  const uint16_t* in;
  const uint16_t* w;   // bf16 [Hq][head_dim][latent_dim]
  uint16_t* out;
  const float* lse_in;  // of the sums' rows, passed on to lse_out (both may be null)
  float* lse_out;
  const LatentRows* rows;
  int32_t num_q_heads;
  LatentRowList list;
};

// Up to 256 cached tokens of a request, for the keys and values of all heads of a group.
constexpr int kLatExpandTok = 256;
struct LatentExpandUnit {
  int32_t x_row;      // first row in the expanded buffers (a multiple of 64)
  int32_t page_base;
  int32_t key0;       // first token (a multiple of kLatExpandTok)
  int32_t key_end;    // tokens of the request; rows past it repeat its last one
  int32_t nrows;      // rows to write, a multiple of 64
  int32_t pad;
};
using LatentExpandList = ShortList<LatentExpandUnit, 96>;

struct LatentExpandParams {
  LatentPoolView pool;
  const uint16_t* w_uk;  // first of the heads
  const uint16_t* w_uv;
  uint16_t* kx;          // bf16 [heads][x_rows][head_dim]
  uint16_t* vx;          // bf16 [heads][x_rows][head_dim]
  uint16_t* rx;          // bf16 [x_rows][64], written with the first group of heads, or null
  const LatentExpandUnit* units;
  int64_t x_rows;
  int32_t heads;
  int32_t heads_per;     // per workgroup (set by the launcher)
  LatentExpandList list;
};

// One workgroup of expanded attention: tokens of one request and head against a range of
// its keys.
struct LatentTile {
  int32_t qo_row;     // suffix row (of the batch) of the tile's first token
  int32_t head_ntok;  // (head within the group << 16) | tokens
  int32_t pos0;       // position of the first token
  int32_t x_row;      // the request's first row in the expanded buffers
  int32_t key_begin;  // multiple of 64
  int32_t key_end;
  int32_t part;       // -1: final result
  int32_t pad;
};
static_assert(sizeof(LatentTile) == 32, "LatentTile is 32 bytes");
constexpr int kLatTileTok = 256;
using LatentTileList = ShortList<LatentTile, 96>;

struct LatentTileMerge {
  int32_t qo_row, head_ntok, part0, nparts;
};
using LatentTileMergeList = ShortList<LatentTileMerge, 96>;

struct LatentPrefillParams {
  const uint16_t* q;   // bf16 [T, Hq, head_dim + 64]
  uint16_t* out;       // bf16 [T, Hq, head_dim]
  float* lse;
  const uint16_t* kx;
  const uint16_t* vx;
  const uint16_t* rx;
  const LatentTile* units;
  float* o_part;       // fp32 [parts][kLatTileTok][head_dim]
  float* lse_part;     // fp32 [parts][kLatTileTok], base 2
  int64_t x_rows;
  int32_t num_q_heads;
  int32_t head0;       // first head of the group
  float scale_log2;
  LatentTileList list;
};

struct LatentTileMergeParams {
  const LatentTileMerge* merges;
  const float* o_part;
  const float* lse_part;
  uint16_t* out;
  float* lse;
  int32_t num_q_heads;
  int32_t head0;
  LatentTileMergeList list;
};
static_assert(sizeof(LatentProjParams) <= 4096 && sizeof(LatentExpandParams) <= 4096 &&
                  sizeof(LatentPrefillParams) <= 4096 && sizeof(LatentTileMergeParams) <= 4096,
              "kernel arguments");

hipError_t launch_latent_absorb(const LatentProjParams& p, int64_t n_rows, int latent_dim, int head_dim,
                                hipStream_t stream);
hipError_t launch_latent_output(const LatentProjParams& p, int64_t n_rows, int latent_dim, int head_dim,
                                hipStream_t stream);
hipError_t launch_latent_expand(const LatentExpandParams& p, int64_t n_units, int latent_dim, int head_dim, bool fp8,
                                hipStream_t stream);
hipError_t launch_latent_prefill(const LatentPrefillParams& p, int64_t n_units, int head_dim, hipStream_t stream);
hipError_t launch_latent_tile_merge(const LatentTileMergeParams& p, int64_t n_merges, int head_dim,
                                    hipStream_t stream);

}  // namespace kvx
