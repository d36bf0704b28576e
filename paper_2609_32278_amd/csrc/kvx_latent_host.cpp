// Host side of latent attention: the C ABI declared in include/kvx_latent.h.
//
// Owns the pool, checks every argument before queuing work, plans the attention of ragged
// (prefix, suffix) pairs over the 256 CUs and their 8 XCDs, and chooses the form of each
// request.

#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <new>
#include <utility>
#include <vector>

#include "kvx_host_util.h"
#include "kvx_latent_internal.h"

using kvx::ceil_div;
using kvx::check_align;
using kvx::check_batch;
using kvx::check_page_ids;
using kvx::hip_fail;
using kvx::LatentExpandUnit;
using kvx::LatentMerge;
using kvx::LatentRows;
using kvx::LatentTile;
using kvx::LatentTileMerge;
using kvx::LatentUnit;
using kvx::report;
using kvx::Staging;
using kvx::Workspace;

struct kvx_latent_pool {
  int device = 0;
  int64_t num_pages = 0;
  int64_t page_bytes = 0;
  int32_t latent_dim = 0;
  int32_t dtype = KVX_LATENT_BF16;
  int32_t split_keys = 0;
  uint8_t* base = nullptr;
  Staging st_rows, st_plan;
  Workspace parts;     // partial results of split key ranges
  Workspace absorbed;  // queries and sums in the latent space
  Workspace expanded;  // keys and values of a group of heads
};

namespace {

constexpr int kSlots = 256;  // CUs, one attention workgroup each
constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kMaxPartBytes = 2ll << 30;
constexpr int64_t kMaxExpandBytes = 2ll << 30;

// Run an entry point's body: no exception crosses the ABI, and an error of the runtime that is
// returned is not left for the caller's next call to find.
template <typename F>
int guarded(F&& body) {
  report(KVX_OK, "%s", "");
  try {
    const int rc = body();
    if (rc == KVX_EHIP || rc == KVX_ENOMEM) (void)hipGetLastError();
    return rc;
  } catch (const std::bad_alloc&) {
    return report(KVX_ENOMEM, "host memory for the plan of the call");
  } catch (...) {
    return report(KVX_EINVAL, "unexpected failure on the host");
  }
}

// The pool's device for the length of a call.
struct OnDevice {
  int before = -1;
  int enter(int device) {
    KVX_HIP(hipGetDevice(&before));
    if (before == device) before = -1;
    else KVX_HIP(hipSetDevice(device));
    return KVX_OK;
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

int check_pool(const kvx_latent_pool* pool) {
  if (pool == nullptr) return report(KVX_EINVAL, "pool is NULL");
  return KVX_OK;
}

int check_stream(hipStream_t s, int device) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  const hipError_t e = hipStreamIsCapturing(s, &st);
  if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
  if (st != hipStreamCaptureStatusNone)
    return report(KVX_EUNSUPPORTED, "the stream is being captured: the plan of a call is made on the host");
  if (s == nullptr || s == hipStreamLegacy || s == hipStreamPerThread) return KVX_OK;  // the current device's
  hipDevice_t of = device;
  KVX_HIP(hipStreamGetDevice(s, &of));
  if (of != device) return report(KVX_EINVAL, "the stream is of device %d, the pool of device %d", of, device);
  return KVX_OK;
}

int check_scale(float sm_scale) {
  if (!(sm_scale > 0.0f) || !std::isfinite(sm_scale * kLog2e))
    return report(KVX_EINVAL, "sm_scale must be > 0 and at most 2e38");
  return KVX_OK;
}

// Heads, rows of one request within an int32, and keys with room for what equal parts, rounded
// up to 64 keys each, go past the last of them (64 keys a part, at most 130560 parts).
constexpr int64_t kMaxKeys = ((int64_t)1 << 31) - ((int64_t)1 << 23);
int check_heads(const kvx_batch* b, int32_t Hq) {
  if (Hq < 1 || Hq > 1024) return report(KVX_EINVAL, "num_q_heads = %d, must be in [1, 1024]", Hq);
  for (int r = 0; r < b->num_reqs; r++) {
    if ((int64_t)b->prefix_lens[r] + b->extend_lens[r] > kMaxKeys)
      return report(KVX_EUNSUPPORTED, "request %d: more than %lld tokens", r, (long long)kMaxKeys);
    if ((int64_t)b->extend_lens[r] * Hq > (int64_t)INT32_MAX - 1024)
      return report(KVX_EUNSUPPORTED, "request %d: %d suffix tokens of %d heads are too many rows", r,
                    b->extend_lens[r], Hq);
  }
  return KVX_OK;
}

// Byte ranges [a, a + n) and [b, b + m) that meet.
bool meet(const void* a, size_t n, const void* b, size_t m) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + m && y < x + n;
}

// Whether [a, a + n) meets one of `rows` rows of `width` bytes, `stride` apart, from b on.
bool meets_rows(const void* a, size_t n, const void* b, int64_t rows, size_t width, size_t stride) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  const uintptr_t i = x < y + width ? 0 : (x - y - width) / stride + 1;  // the first row that ends behind x
  return i < (uintptr_t)rows && y + i * stride < x + n;
}

// The results of attention, over rows of `row` bytes each, against what it reads and each other.
int check_results(const void* out, size_t row, const float* lse, size_t rows, const void* q, size_t q_row,
                  const void* w_uk = nullptr, const void* w_uv = nullptr, size_t w_bytes = 0) {
  if (meet(out, rows * row, q, rows * q_row) || meet(out, rows * row, w_uk, w_bytes) || meet(out, rows * row, w_uv, w_bytes))
    return report(KVX_EINVAL, "out overlaps an input");
  if (lse == nullptr) return KVX_OK;
  const size_t n = rows * sizeof(float);
  if (meet(lse, n, q, rows * q_row) || meet(lse, n, w_uk, w_bytes) || meet(lse, n, w_uv, w_bytes))
    return report(KVX_EINVAL, "lse overlaps an input");
  if (meet(lse, n, out, rows * row)) return report(KVX_EINVAL, "lse overlaps out");
  return KVX_OK;
}

kvx::LatentPoolView view(const kvx_latent_pool* pool, const kvx_batch* batch) {
  return {pool->base, pool->page_bytes, batch->page_ids};
}

// The touched pages of a batch's suffixes, request by request.
std::vector<kvx::RopeUnit> page_units(const kvx_batch* batch, const std::vector<int64_t>& qo) {
  std::vector<kvx::RopeUnit> units;
  const int64_t S = kvx::kPageSize;
  for (int r = 0; r < batch->num_reqs; r++) {
    const int64_t P = batch->prefix_lens[r], E = batch->extend_lens[r], L = P + E;
    if (E == 0) continue;
    for (int64_t lp = P / S; lp <= (L - 1) / S; lp++) {
      kvx::RopeUnit u;
      u.row_slot0 = (int32_t)(qo[(size_t)r] + lp * S - P);
      u.page_pos = (int32_t)(batch->page_indptr[r] + lp);
      u.slot_begin = (int32_t)(std::max<int64_t>(P, lp * S) - lp * S);
      u.slot_end = (int32_t)(std::min<int64_t>(L, lp * S + S) - lp * S);
      u.pos_slot0 = (int32_t)(lp * S);
      units.push_back(u);
    }
  }
  return units;
}

// The units of a store or load call, in its arguments or uploaded.
template <typename Params>
int place_units(kvx_latent_pool* pool, const kvx_batch* batch, const std::vector<int64_t>& qo, hipStream_t s,
                Params& p, int64_t& n_units) {
  p.units = nullptr;
  if (kvx::inline_store_reqs(batch, qo, p.reqs)) {
    n_units = p.reqs.first[p.reqs.n];
    return KVX_OK;
  }
  const std::vector<kvx::RopeUnit> units = page_units(batch, qo);
  n_units = (int64_t)units.size();
  void* dev = nullptr;
  if (int rc = pool->st_rows.upload(units.data(), units.size() * sizeof(kvx::RopeUnit), s, &dev)) return rc;
  p.units = (const kvx::RopeUnit*)dev;
  return KVX_OK;
}

int check_stride(int64_t stride, int row, const char* name) {
  if (stride < row || stride % 8 != 0 || stride > (int64_t)1 << 40)
    return report(KVX_EINVAL, "%s = %lld: must be a multiple of 8, at least %d", name, (long long)stride, row);
  return KVX_OK;
}

int store_call(kvx_latent_pool* pool, const kvx_batch* batch, const kvx_rope* rope, bool rotate, const void* q,
               int32_t Hq, int32_t q_dim, void* q_out, const void* kv, int64_t kv_stride, hipStream_t s) {
  if (int rc = check_pool(pool)) return rc;
  std::vector<int64_t> qo;
  if (int rc = check_batch(batch, qo)) return rc;
  kvx::LatentStoreParams p{};
  bool interleaved = false;
  if (rotate) {
    if (rope == nullptr) return report(KVX_EINVAL, "rope is NULL");
    if (rope->rotary_dim != kvx::kLatRope)
      return report(KVX_EINVAL, "rotary_dim = %d, must be the pool's rope_dim = %d", rope->rotary_dim, kvx::kLatRope);
    if (rope->style != KVX_ROPE_HALF && rope->style != KVX_ROPE_INTERLEAVED)
      return report(KVX_EINVAL, "style = %d", rope->style);
    if (!(rope->norm_eps >= 0.0f) || !std::isfinite(rope->norm_eps))
      return report(KVX_EINVAL, "norm_eps must be finite and >= 0");
    if (rope->q_norm != nullptr) return report(KVX_EINVAL, "q_norm must be NULL");
    if (int rc = check_align(rope->k_norm, "k_norm")) return rc;
    for (int j = 0; j < kvx::kLatRope / 2; j++) {
      double f;
      if (rope->inv_freq) {
        f = rope->inv_freq[j];
        if (!(f >= 0.0) || !std::isfinite(f)) return report(KVX_EINVAL, "inv_freq[%d] must be finite and >= 0", j);
      } else {
        if (!(rope->theta > 0.0) || !std::isfinite(rope->theta))
          return report(KVX_EINVAL, "theta must be finite and > 0");
        f = std::pow(rope->theta, -2.0 * j / kvx::kLatRope);
      }
      p.rev_freq[j] = f / 6.283185307179586476925286766559;  // turns per position
    }
    interleaved = rope->style == KVX_ROPE_INTERLEAVED;
    if (Hq < 0 || Hq > 1024) return report(KVX_EINVAL, "num_q_heads = %d, must be in [0, 1024]", Hq);
    if (Hq > 0) {
      if (!q || !q_out) return report(KVX_EINVAL, "q and q_out must be non-NULL");
      if (q_dim < kvx::kLatRope || q_dim > 4096 || q_dim % 8 != 0)
        return report(KVX_EINVAL, "q_dim = %d: must be a multiple of 8 in [%d, 4096]", q_dim, kvx::kLatRope);
      if (int rc = check_align(q, "q")) return rc;
      if (int rc = check_align(q_out, "q_out")) return rc;
      const size_t q_bytes = (size_t)qo.back() * Hq * q_dim * 2;
      if (q != q_out && meet(q, q_bytes, q_out, q_bytes))
        return report(KVX_EINVAL, "q_out overlaps q without being q");
    }
    p.norm = (const uint16_t*)rope->k_norm;
    p.norm_eps = rope->norm_eps;
    p.rotate = 1;
  }
  if (int rc = check_stride(kv_stride, pool->latent_dim + kvx::kLatRope, "kv_stride")) return rc;
  if (int rc = check_align(kv, "kv")) return rc;
  if (qo.back() == 0) return KVX_OK;
  if (!kv) return report(KVX_EINVAL, "kv is NULL");
  if (rotate && Hq > 0 && meets_rows(q_out, (size_t)qo.back() * Hq * q_dim * 2, kv, qo.back(),
                                     (size_t)(pool->latent_dim + kvx::kLatRope) * 2, (size_t)kv_stride * 2))
    return report(KVX_EINVAL, "q_out overlaps kv");
  OnDevice on;
  if (int rc = on.enter(pool->device)) return rc;
  if (int rc = check_stream(s, pool->device)) return rc;
  if (kvx::validate_mode())
    if (int rc = check_page_ids(pool->num_pages, batch, s)) return rc;
  int64_t n_units = 0;
  if (int rc = place_units(pool, batch, qo, s, p, n_units)) return rc;
  p.pool = view(pool, batch);
  p.kv = (const uint16_t*)kv;
  p.kv_stride = kv_stride;
  p.q = (const uint16_t*)q;
  p.q_out = (uint16_t*)q_out;
  p.num_q_heads = Hq;
  p.q_dim = q_dim;
  const hipError_t e =
      kvx::launch_store_latent(p, n_units, pool->latent_dim, pool->dtype == KVX_LATENT_FP8, interleaved, s);
  if (e != hipSuccess) return hip_fail(e, "store_latent kernel launch");
  return p.units ? pool->st_rows.done(s) : KVX_OK;
}

// ------------------------------------------------------------------ plans

// Host arrays of a call, uploaded in one piece.
struct Blob {
  std::vector<uint8_t> bytes;
  template <typename U>
  size_t add(const std::vector<U>& v) {
    bytes.resize((bytes.size() + 15) / 16 * 16);
    const size_t at = bytes.size();
    bytes.resize(at + v.size() * sizeof(U));
    if (!v.empty()) std::memcpy(bytes.data() + at, v.data(), v.size() * sizeof(U));
    return at;
  }
};

// A list for the arguments of its kernel, or added to the blob; returns its offset there.
template <typename U, int N>
size_t place_list(const std::vector<U>& v, kvx::ShortList<U, N>& list, Blob& blob) {
  list.n = 0;
  if (v.size() > (size_t)N) return blob.add(v);
  list.n = (int32_t)v.size();
  std::copy(v.begin(), v.end(), list.at);
  return 0;
}

// Work that shares its keys, to run on one XCD: units [first, first + count), each of them
// `cost` long at most.
struct Group {
  double cost;
  int32_t first, count;
};

// Launch order (workgroup i runs on XCD i % 8): groups, longest first, each to the XCD that has
// the CU which is free first; -1 pads the shorter queues.
std::vector<int32_t> spread(std::vector<Group>& groups) {
  // A group that is a large share of all would leave other XCDs idle: no more than a 64th of
  // the units stay together.
  int64_t units = 0;
  for (const Group& g : groups) units += g.count;
  const int32_t most_units = (int32_t)std::max<int64_t>(1, units / 64);
  for (size_t i = 0, n = groups.size(); i < n; i++) {
    while (groups[i].count > most_units) {
      groups[i].count -= most_units;
      const Group rest{groups[i].cost, groups[i].first + groups[i].count, most_units};
      groups.push_back(rest);
    }
  }
  std::stable_sort(groups.begin(), groups.end(), [](const Group& a, const Group& b) { return a.cost > b.cost; });
  constexpr int kXcds = kvx::kNumXcd, kCus = kSlots / kXcds;
  struct Xcd {
    double free[kCus] = {};  // when its CUs are, a heap with the earliest first
    std::vector<int32_t> queue;
  };
  Xcd xcd[kXcds];
  for (const Group& g : groups) {
    // the XCD, and on it as many units as have a CU at about the time that its first has
    for (int32_t at = 0; at < g.count;) {
      Xcd* x = &xcd[0];
      for (Xcd& y : xcd)
        if (y.free[0] < x->free[0] || (y.free[0] == x->free[0] && y.queue.size() < x->queue.size())) x = &y;
      const double limit = x->free[0] + 0.1 * g.cost;
      do {
        std::pop_heap(x->free, x->free + kCus, std::greater<double>());
        x->free[kCus - 1] += g.cost;
        std::push_heap(x->free, x->free + kCus, std::greater<double>());
        x->queue.push_back(g.first + at++);
      } while (at < g.count && x->free[0] <= limit);
    }
  }
  size_t most = 0;
  for (const Xcd& x : xcd) most = std::max(most, x.queue.size());
  std::vector<int32_t> out(most * kXcds, -1);
  for (size_t x = 0; x < (size_t)kXcds; x++)
    for (size_t i = 0; i < xcd[x].queue.size(); i++) out[i * kXcds + x] = xcd[x].queue[i];
  while (!out.empty() && out.back() < 0) out.pop_back();
  return out;
}

template <typename U>
std::vector<U> in_order(const std::vector<U>& units, const std::vector<int32_t>& order) {
  std::vector<U> out(order.size());  // value-initialised: padding
  for (size_t i = 0; i < order.size(); i++)
    if (order[i] >= 0) out[i] = units[(size_t)order[i]];
  return out;
}

// What a plan's length search sees of a request: `tiles` tiles of rows over about `len` steps
// of 64 keys each.
struct Span {
  int64_t tiles, len;
};

// Parts of at most `steps` steps of 64 keys (0: nothing is split): of equal length, or, where a
// length was asked for, `cut` every `steps`.
struct Split {
  int64_t steps = 0;
  bool cut = false;
  int64_t parts(int64_t len) const { return steps > 0 ? ceil_div(len, steps) : 1; }
  int64_t part_len(int64_t len) const { return cut && parts(len) > 1 ? steps : ceil_div(len, parts(len)); }
};

// What a unit costs besides its steps of 64 keys, in such steps: its first loads and its
// epilogue; the result of a part, written and read again.  Fitted to four batches of 64-row
// units timed at ten forced lengths each (a step is 1.8 us).  Smaller units have less to load
// and to write.
struct UnitCosts {
  double start, part;
};

// Estimated time of a plan: units, longest first, each to the CU that is free first.  Equal CUs
// are kept together, a plan of very many units counts as even, and the search stops beyond
// `limit`, as planning is on the path of every call.
double plan_time(const std::vector<Span>& spans, const Split& split, const UnitCosts& k, double limit) {
  double total = 0.0, top = 0.0;
  int64_t units = 0, most = 1;
  auto cost = [&](const Span& s) {
    return (double)split.part_len(s.len) + k.start + (split.parts(s.len) > 1 ? k.part : 0.0);
  };
  for (const Span& s : spans) {
    const int64_t parts = split.parts(s.len);
    total += cost(s) * (double)(s.tiles * parts);
    units += s.tiles * parts;
    top = std::max(top, cost(s));
    most = std::max(most, parts);
  }
  const double merge = most > 1 ? 2.0 + 0.12 * (double)most : 0.0;
  const double least = std::max(top, total / kSlots) + merge;
  if (least >= limit || units <= kSlots) return least;
  if (units > 3 * kSlots) return std::max(top, total / kSlots + 0.5 * top) + merge;
  using Work = std::pair<double, int64_t>;  // cost, units; or free at, CUs
  std::vector<Work> work;
  for (const Span& s : spans) work.push_back({cost(s), s.tiles * split.parts(s.len)});
  std::sort(work.begin(), work.end(), std::greater<Work>());
  std::vector<Work> cus{{0.0, kSlots}};  // a heap with the earliest first
  double end = 0.0;
  for (Work& w : work) {
    while (w.second > 0) {
      std::pop_heap(cus.begin(), cus.end(), std::greater<Work>());
      Work& c = cus.back();
      const double from = c.first;
      const int64_t n = std::min(w.second, c.second), left = c.second - n;
      c = {from + w.first, n};
      std::push_heap(cus.begin(), cus.end(), std::greater<Work>());
      if (left > 0) {
        cus.push_back({from, left});
        std::push_heap(cus.begin(), cus.end(), std::greater<Work>());
      }
      end = std::max(end, from + w.first);
      w.second -= n;
    }
    if (end + merge >= limit) break;
  }
  return end + merge;
}

// A dozen forced lengths from 512 to 16384 keys against this choice, whole calls in us, best forced
// length in brackets: decode of 128 requests on 16 heads 339 (352), 24 long requests on 128
// heads 442 (434), drafts of 32 requests 175 (162, a length that fits this batch by chance),
// short turns 655 (675).
Split choose_split(const std::vector<Span>& spans, const UnitCosts& k) {
  int64_t work = 0, longest = 0;
  for (const Span& s : spans) {
    work += s.tiles * s.len;
    longest = std::max(longest, s.len);
  }
  Split best;
  if (work == 0) return best;
  double at = plan_time(spans, best, k, HUGE_VAL);
  for (const double rounds : {0.9, 1.0, 0.75, 0.5, 0.25, 1.2, 1.5, 1.75, 2.0, 2.5, 3.0, 4.0, 6.0}) {
    const int64_t c = std::max<int64_t>(1, (int64_t)std::ceil((double)work / (rounds * kSlots)));
    if (c >= longest) continue;
    const double t = plan_time(spans, Split{c}, k, at);
    if (t < at) {
      at = t;
      best = Split{c};
    }
  }
  return best;
}

// Longer parts where there would be more of them than `most`.
void bound_parts(const std::vector<Span>& spans, int64_t most, Split& split) {
  while (split.steps > 0) {
    int64_t n = 0;
    for (const Span& s : spans)
      if (split.parts(s.len) > 1) n += s.tiles * split.parts(s.len);
    if (n <= most) return;
    split.steps *= 2;
  }
}

struct AbsorbedPlan {
  std::vector<LatentUnit> units;
  std::vector<LatentMerge> merges;
  int64_t n_parts = 0;
  int row_blocks = 1;
  bool in_args = false;  // `rows` (rows.n > 0) or `small` holds the plan instead
  kvx::LatentRowPlan rows;
  kvx::LatentSmallPlan small;
};

// One request of the absorbed form: its batch index and the row that its first suffix token
// has in the arrays the attention works on.
struct Member {
  int32_t req;
  int64_t row;
};

void plan_absorbed(const kvx_batch* b, const std::vector<Member>& members, int32_t Hq, int32_t latent_dim,
                   int32_t split_keys, AbsorbedPlan& plan) {
  int64_t most = 0;
  for (const Member& m : members) most = std::max<int64_t>(most, (int64_t)b->extend_lens[m.req] * Hq);
  // Rows of a unit, as many as the request with the most rows fills.  With 16, 32 and 64 rows:
  // 128 requests of one token, 4k to 32k keys, 16 heads 361, 373, 391 us; 32 heads 520, 378, 396
  // (8 bits 344, 241, 306); 4 requests on 1k to 8k keys, 16 heads 19.8, 21.8, 24.5; 32 of them, 24
  // heads 48.7, 34.9, 37.8.  Requests of many rows read their keys once a unit.
  plan.row_blocks = most <= 16 ? 1 : (most <= 32 ? 2 : 4);
  const int64_t M = 16 * plan.row_blocks;
  std::vector<Span> spans;
  for (const Member& m : members) {
    const int64_t E = b->extend_lens[m.req], L = b->prefix_lens[m.req] + E;
    spans.push_back({ceil_div(E * Hq, M), ceil_div(L, kvx::kLatTileKeys)});
  }
  Split split{split_keys / kvx::kLatTileKeys, true};
  const UnitCosts costs = plan.row_blocks == 4 ? UnitCosts{6.0, 6.0} : UnitCosts{4.0, 2.0};
  if (split_keys == 0) split = choose_split(spans, costs);
  bound_parts(spans, kMaxPartBytes / (M * (latent_dim + 1) * 4), split);
  const int32_t R = (int32_t)members.size();
  plan.rows.n = 0;
  if (R <= kvx::kLatRowReqs && std::all_of(spans.begin(), spans.end(), [](const Span& s) { return s.tiles == 1; })) {
    // longest parts first
    std::vector<int32_t> by(members.size());
    std::vector<int64_t> len(members.size());
    for (int32_t i = 0; i < R; i++) {
      by[(size_t)i] = i;
      len[(size_t)i] = split.part_len(spans[(size_t)i].len);
    }
    std::stable_sort(by.begin(), by.end(), [&](int32_t a, int32_t b) { return len[(size_t)a] > len[(size_t)b]; });
    kvx::LatentRowPlan& rp = plan.rows;
    int64_t at = 0;
    bool merges = false;
    for (int32_t i = 0; i < R; i++) {
      const Member& m = members[(size_t)by[(size_t)i]];
      const int64_t keys = (int64_t)b->prefix_lens[m.req] + b->extend_lens[m.req];
      const int64_t l = len[(size_t)by[(size_t)i]] * kvx::kLatTileKeys, parts = ceil_div(keys, l);
      rp.first[i] = (int32_t)at;
      rp.qo[i] = (int32_t)m.row;
      rp.extend[i] = b->extend_lens[m.req];
      rp.prefix[i] = b->prefix_lens[m.req];
      rp.page_base[i] = b->page_indptr[m.req];
      rp.len[i] = (int32_t)l;
      rp.part0[i] = (int32_t)plan.n_parts;
      at += parts;
      if (parts > 1) plan.n_parts += parts, merges = true;
    }
    std::fill(rp.first + R, rp.first + kvx::kLatRowReqs, INT32_MAX);
    rp.n = R;
    rp.n_units = (int32_t)at;
    plan.in_args = true;
    if (merges) plan.merges.resize(1);  // a merge launch is needed
    return;
  }
  std::vector<LatentUnit> units;
  std::vector<uint16_t> codes;  // of the units, while the plan may be a small one
  std::vector<Group> groups;
  int64_t all_tiles = 0, most_parts = 1;
  for (const Span& s : spans) all_tiles += s.tiles, most_parts = std::max(most_parts, split.parts(s.len));
  bool small = all_tiles <= kvx::kLatSmallTiles && most_parts <= kvx::kLatSmallParts;
  int32_t n_tiles = 0;
  for (size_t i = 0; i < members.size(); i++) {
    const Member& m = members[i];
    const int64_t P = b->prefix_lens[m.req], E = b->extend_lens[m.req], rows = E * Hq;
    const int64_t parts = split.parts(spans[i].len), len = split.part_len(spans[i].len) * kvx::kLatTileKeys;
    const int64_t part0 = plan.n_parts;
    const int64_t tiles = spans[i].tiles;
    if (parts > 1) plan.n_parts += tiles * parts;
    if (small) {
      for (int64_t t = 0; t < tiles; t++) {
        const int64_t n = std::min<int64_t>(M, rows - t * M);
        plan.small.tile[n_tiles + t] = {(int32_t)(t * M), (int32_t)n, (int32_t)m.row, (int32_t)P,
                                        b->page_indptr[m.req], (int32_t)(P + (t * M + n - 1) / Hq + 1), (int32_t)len,
                                        (int32_t)(part0 + t * parts)};
      }
    }
    for (int64_t c = 0; c < parts; c++) {
      Group g{0.0, (int32_t)units.size(), 0};
      for (int64_t t = tiles - 1; t >= 0; t--) {
        LatentUnit u{};
        u.row0 = (int32_t)(t * M);
        u.nrows = (int32_t)std::min<int64_t>(M, rows - t * M);
        u.qo = (int32_t)m.row;
        u.prefix = (int32_t)P;
        u.page_base = b->page_indptr[m.req];
        const int64_t end = P + (u.row0 + u.nrows - 1) / Hq + 1;  // keys that a row of the tile sees
        if (c * len >= end) continue;
        u.key_begin = (int32_t)(c * len);
        u.key_end = (int32_t)std::min<int64_t>(end, (c + 1) * len);
        u.part = end > len ? (int32_t)(part0 + t * parts + c) : -1;
        g.cost = std::max(g.cost, (double)ceil_div(u.key_end - u.key_begin, kvx::kLatTileKeys) + costs.start +
                                      (u.part >= 0 ? costs.part : 0.0));
        units.push_back(u);
        if (small) codes.push_back((uint16_t)((n_tiles + t) << 10 | c));
        g.count++;
        if (c == 0 && end > len) {
          const int64_t n = ceil_div(end, len);
          plan.merges.push_back({u.row0, u.nrows, u.qo, (int32_t)(part0 + t * parts), (int32_t)n, 0});
        }
      }
      if (g.count > 0) groups.push_back(g);
    }
    n_tiles += (int32_t)tiles;
  }
  const std::vector<int32_t> order = spread(groups);
  plan.in_args = small && order.size() <= (size_t)kvx::kLatSmallUnits;
  if (!plan.in_args) {
    plan.units = in_order(units, order);
    return;
  }
  plan.small.n_units = (int32_t)order.size();
  plan.small.n_tiles = n_tiles;
  for (size_t i = 0; i < order.size(); i++)
    plan.small.code[i] = order[i] < 0 ? kvx::kLatNoUnit : codes[(size_t)order[i]];
}

struct ExpandedPlan {
  std::vector<LatentExpandUnit> expand;
  std::vector<LatentTile> units;
  std::vector<LatentTileMerge> merges;
  int64_t n_parts = 0;
};

// Rows of the expanded buffers: requests side by side, each from a multiple of 64.
int64_t expand_units(const kvx_batch* b, const std::vector<int32_t>& reqs, std::vector<LatentExpandUnit>& out,
                     std::vector<int64_t>& x_row) {
  int64_t at = 0;
  for (int32_t r : reqs) {
    const int64_t L = (int64_t)b->prefix_lens[r] + b->extend_lens[r];
    x_row.push_back(at);
    const int64_t rows = ceil_div(L, 64) * 64;
    for (int64_t k = 0; k < rows; k += kvx::kLatExpandTok)
      out.push_back({(int32_t)(at + k), b->page_indptr[r], (int32_t)k, (int32_t)L,
                     (int32_t)std::min<int64_t>(kvx::kLatExpandTok, rows - k), 0});
    at += rows;
  }
  return at;
}

void plan_expanded(const kvx_batch* b, const std::vector<int64_t>& qo, const std::vector<int32_t>& reqs,
                   const std::vector<int64_t>& x_row, int32_t heads, int32_t head_dim, ExpandedPlan& plan) {
  const int64_t M = kvx::kLatTileTok;
  std::vector<Span> spans;
  for (int32_t r : reqs) {
    const int64_t E = b->extend_lens[r], L = b->prefix_lens[r] + E;
    spans.push_back({ceil_div(E, M) * heads, ceil_div(b->prefix_lens[r] + L, 128)});  // of its tiles on average
  }
  const UnitCosts costs{6.0, 6.0};
  Split split = choose_split(spans, costs);
  // of the longest tiles, which the parts are made for
  std::vector<Span> longest;
  for (size_t i = 0; i < reqs.size(); i++)
    longest.push_back({spans[i].tiles, ceil_div((int64_t)b->prefix_lens[reqs[i]] + b->extend_lens[reqs[i]], 64)});
  bound_parts(longest, kMaxPartBytes / (M * (head_dim + 1) * 4), split);
  std::vector<LatentTile> units;
  std::vector<Group> groups;
  for (size_t i = 0; i < reqs.size(); i++) {
    const int32_t r = reqs[i];
    const int64_t P = b->prefix_lens[r], E = b->extend_lens[r], tiles = ceil_div(E, M);
    const int64_t parts = split.parts(longest[i].len), len = split.part_len(longest[i].len) * 64;
    for (int32_t h = 0; h < heads; h++) {
      const int64_t part0 = plan.n_parts;
      if (parts > 1) plan.n_parts += tiles * parts;
      for (int64_t c = 0; c < parts; c++) {
        Group g{0.0, (int32_t)units.size(), 0};
        for (int64_t t = tiles - 1; t >= 0; t--) {
          const int64_t n = std::min<int64_t>(M, E - t * M), end = P + t * M + n;
          if (c * len >= end) continue;
          LatentTile u{};
          u.qo_row = (int32_t)(qo[(size_t)r] + t * M);
          u.head_ntok = (int32_t)(h << 16 | n);
          u.pos0 = (int32_t)(P + t * M);
          u.x_row = (int32_t)x_row[i];
          u.key_begin = (int32_t)(c * len);
          u.key_end = (int32_t)std::min<int64_t>(end, (c + 1) * len);
          u.part = end > len ? (int32_t)(part0 + t * parts + c) : -1;
          g.cost = std::max(g.cost, (double)ceil_div(u.key_end - u.key_begin, 64) + costs.start +
                                        (u.part >= 0 ? costs.part : 0.0));
          units.push_back(u);
          g.count++;
          if (c == 0 && end > len)
            plan.merges.push_back({u.qo_row, u.head_ntok, (int32_t)(part0 + t * parts), (int32_t)ceil_div(end, len)});
        }
        if (g.count > 0) groups.push_back(g);
      }
    }
  }
  plan.units = in_order(units, spread(groups));
}

// Rows of the expanded buffers for the requests that do not take the absorbed form.
int64_t tokens_to_expand(const kvx_batch* b, const std::vector<bool>& absorbed) {
  int64_t n = 0;
  for (int32_t r = 0; r < b->num_reqs; r++)
    if (b->extend_lens[r] > 0 && !absorbed[(size_t)r])
      n += ceil_div((int64_t)b->prefix_lens[r] + b->extend_lens[r], 64) * 64;
  return n;
}

// The requests of a batch that take the absorbed form, by the estimated time of each form: what
// its kernels compute (suffixes in whole units of 16, 32 or 64 rows, or tiles of 256 tokens,
// cached tokens expanded 256 at a time) at the rates that they reach, what a unit costs besides,
// and the launches with one unit's walk along its keys, which few units do not hide.  All of one
// form, or each request its cheaper one.
// Fitted to both forms' times at 14 suffix lengths from 1 to 700 of 32 batches (latent 256 and 512,
// heads of 64 and 128, both pool types), in us absorbed / expanded: 12 requests of 8000 cached
// tokens and 16 heads, latent 512, heads of 128, 128 new tokens 471 / 674, 257 956 / 935, 512
// 1545 / 980; 8 bits 519 / 652, 1138 / 906, 1775 / 954; latent 256, heads of 64 288 / 339, 604 / 486,
// 932 / 512; and of 550 random batches.  400 other random batches: on average 1.6% above the
// faster of the two, at most 1.4 times, where both are some 25 us (by the pairs alone, without
// whole tiles and units, their start and steps: 17%, 4.7 times; 23 short requests of 102 heads
// 112 us where 42 do).
std::vector<bool> choose_forms(const kvx_batch* b, int32_t Hq, int64_t latent, int64_t d, bool fp8 = false) {
  // operations a us
  const double rate_a = (latent == 512 ? 1.28e9 : 1.0e9) * (fp8 ? 0.84 : 1.0), rate_weights = 0.45e9;
  const double rate_e = d == 128 ? 1.06e9 : 0.85e9, rate_expand = 1.28e9;
  // what a unit costs besides, in steps of 64 keys
  constexpr double kUnitA = 14.0, kUnitE = 4.3;
  constexpr int64_t T = kvx::kLatTileTok;
  const int32_t R = b->num_reqs;
  int64_t most = 0, longest = 0;
  for (int32_t r = 0; r < R; r++)
    if (b->extend_lens[r] > 0) {
      most = std::max<int64_t>(most, (int64_t)b->extend_lens[r] * Hq);
      longest = std::max<int64_t>(longest, (int64_t)b->prefix_lens[r] + b->extend_lens[r]);
    }
  const int64_t M = most <= 16 ? 16 : (most <= 32 ? 32 : 64);  // rows of the absorbed form's units
  // us of launches and of the steps of one unit (a longer walk is split between more units)
  const double steps = (double)ceil_div(std::min<int64_t>(longest, 1024), kvx::kLatTileKeys);
  const double wide = latent / 512.0;
  const double start_a = 21.0 + (M == 64 ? 9.0 * wide : 0.0) + 1.1 * wide * (M == 64 && fp8 ? 1.2 : 1.0) * steps;
  const double start_e = 16.0 + 3.0 * wide + 2.4 * d / 128.0 * steps;
  std::vector<bool> absorbed((size_t)R);
  double all_a = start_a, all_e = start_e, mixed = start_a + start_e;
  for (int32_t r = 0; r < R; r++) {
    const int64_t P = b->prefix_lens[r], E = b->extend_lens[r];
    if (E == 0) continue;
    // pairs: a unit's or tile's rows see the keys up to its last token's
    const double keys_a = P + 0.5 * (E + (double)M / Hq) + kUnitA * kvx::kLatTileKeys;
    const double keys_e = P + 0.5 * (E + std::min(E, T)) + kUnitE * kvx::kLatTileKeys;
    const double pairs_a = (double)(ceil_div(E * Hq, M) * M) * keys_a, pairs_e = (double)(ceil_div(E, T) * T * Hq) * keys_e;
    const double weights = 4.0 * d * latent * Hq;  // operations a token
    const double a = 2.0 * (2.0 * latent + kvx::kLatRope) * pairs_a / rate_a + weights * E / rate_weights;
    const double e = 2.0 * (2.0 * d + kvx::kLatRope) * pairs_e / rate_e +
                     weights * (double)(ceil_div(P + E, kvx::kLatExpandTok) * kvx::kLatExpandTok) / rate_expand;
    absorbed[(size_t)r] = a <= e;
    all_a += a;
    all_e += e;
    mixed += std::min(a, e);
  }
  if (all_a <= mixed || all_e <= mixed) absorbed.assign((size_t)R, all_a <= all_e);
  if (tokens_to_expand(b, absorbed) > INT32_MAX) absorbed.assign((size_t)R, true);
  return absorbed;
}

// Attention on latents over `members`: launches its kernel and merge; the plan is at `dev`.
int launch_absorbed(kvx_latent_pool* pool, const kvx_batch* batch, const AbsorbedPlan& plan, const uint8_t* dev,
                    size_t units_at, size_t merges_at, const void* q, int32_t Hq, float sm_scale, void* out,
                    float* lse, hipStream_t s) {
  kvx::LatentAttnParams p{};
  p.pool = view(pool, batch);
  p.q = (const uint16_t*)q;
  p.out = (uint16_t*)out;
  p.lse = lse;
  p.units = (const LatentUnit*)(dev + units_at);
  const size_t per_part = (size_t)16 * plan.row_blocks * pool->latent_dim;
  if (plan.n_parts > 0) {
    if (int rc = pool->parts.ensure((size_t)plan.n_parts * (per_part + 16 * plan.row_blocks) * sizeof(float), s))
      return rc;
    p.o_part = (float*)pool->parts.ptr;
    p.lse_part = p.o_part + (size_t)plan.n_parts * per_part;
  }
  p.num_q_heads = Hq;
  p.scale_log2 = sm_scale * kLog2e;
  const kvx::LatentRowPlan* rows = plan.in_args && plan.rows.n > 0 ? &plan.rows : nullptr;
  const kvx::LatentSmallPlan* small = plan.in_args && !rows ? &plan.small : nullptr;
  hipError_t e = kvx::launch_latent_attention(p, (int64_t)plan.units.size(), small, rows, pool->latent_dim,
                                              pool->dtype == KVX_LATENT_FP8, plan.row_blocks, s);
  if (e != hipSuccess) return hip_fail(e, "latent attention kernel launch");
  if (!plan.merges.empty()) {
    kvx::LatentMergeParams m{};
    m.merges = (const LatentMerge*)(dev + merges_at);
    m.o_part = p.o_part;
    m.lse_part = p.lse_part;
    m.out = p.out;
    m.lse = lse;
    m.num_q_heads = Hq;
    e = kvx::launch_latent_merge(m, (int64_t)plan.merges.size(), small, rows, pool->latent_dim, plan.row_blocks, s);
    if (e != hipSuccess) return hip_fail(e, "latent merge kernel launch");
  }
  return plan.n_parts > 0 ? pool->parts.done(s) : KVX_OK;
}

}  // namespace

extern "C" {

int latent_pool_create(int64_t num_pages, int32_t page_size, int32_t latent_dim, int32_t rope_dim, int32_t dtype,
                       kvx_latent_pool** out) {
  return guarded([&]() -> int {
    if (out == nullptr) return report(KVX_EINVAL, "out is NULL");
    *out = nullptr;
    if (num_pages <= 0 || num_pages > (int64_t)INT32_MAX)
      return report(KVX_EINVAL, "num_pages = %lld must be in [1, 2^31-1]", (long long)num_pages);
    if (page_size != kvx::kPageSize) return report(KVX_EUNSUPPORTED, "page_size %d (supported: 16)", page_size);
    if (latent_dim != 256 && latent_dim != 512)
      return report(KVX_EUNSUPPORTED, "latent_dim %d (supported: 256, 512)", latent_dim);
    if (rope_dim != kvx::kLatRope) return report(KVX_EUNSUPPORTED, "rope_dim %d (supported: 64)", rope_dim);
    if (dtype != KVX_LATENT_BF16 && dtype != KVX_LATENT_FP8) return report(KVX_EINVAL, "dtype %d", dtype);
    kvx_latent_pool* p = new kvx_latent_pool();
    p->num_pages = num_pages;
    p->latent_dim = latent_dim;
    p->dtype = dtype;
    p->page_bytes = kvx::kPageSize * (dtype == KVX_LATENT_FP8
                                          ? (int64_t)latent_dim + 2 * rope_dim + latent_dim / kvx::kLatGroup
                                          : 2 * ((int64_t)latent_dim + rope_dim));
    hipError_t e = hipGetDevice(&p->device);
    if (e == hipSuccess) e = hipMalloc((void**)&p->base, (size_t)num_pages * p->page_bytes);
    if (e == hipSuccess) e = hipMemset(p->base, 0, (size_t)num_pages * p->page_bytes);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
      if (p->base) (void)hipFree(p->base);
      delete p;
      return hip_fail(e, "latent pool allocation");
    }
    *out = p;
    return KVX_OK;
  });
}

int latent_pool_destroy(kvx_latent_pool* pool) {
  return guarded([&]() -> int {
    if (pool == nullptr) return KVX_OK;
    OnDevice on;
    (void)on.enter(pool->device);
    const hipError_t e = hipDeviceSynchronize();
    pool->st_rows.release();
    pool->st_plan.release();
    pool->parts.release();
    pool->absorbed.release();
    pool->expanded.release();
    if (pool->base) (void)hipFree(pool->base);
    delete pool;
    if (e != hipSuccess) return hip_fail(e, "hipDeviceSynchronize");
    return KVX_OK;
  });
}

int latent_pool_layout(const kvx_latent_pool* pool, kvx_latent_layout* out) {
  return guarded([&]() -> int {
    if (int rc = check_pool(pool)) return rc;
    if (out == nullptr) return report(KVX_EINVAL, "out is NULL");
    std::memset(out, 0, sizeof *out);
    out->base = pool->base;
    out->num_pages = pool->num_pages;
    out->page_bytes = pool->page_bytes;
    out->page_size = kvx::kPageSize;
    out->latent_dim = pool->latent_dim;
    out->rope_dim = kvx::kLatRope;
    out->dtype = pool->dtype;
    const bool fp8 = pool->dtype == KVX_LATENT_FP8;
    out->key_offset = fp8 ? kvx::kPageSize * pool->latent_dim : 2 * pool->latent_dim;
    out->scale_offset = fp8 ? kvx::kPageSize * (pool->latent_dim + 2 * kvx::kLatRope) : 0;
    return KVX_OK;
  });
}

int latent_pool_set_split_keys(kvx_latent_pool* pool, int32_t keys) {
  return guarded([&]() -> int {
    if (int rc = check_pool(pool)) return rc;
    if (keys < 0 || keys % kvx::kLatTileKeys != 0)
      return report(KVX_EINVAL, "split keys %d: must be 0 or a positive multiple of %d", keys, kvx::kLatTileKeys);
    pool->split_keys = keys;
    return KVX_OK;
  });
}

int store_latent(kvx_latent_pool* pool, const kvx_batch* batch, const void* kv, int64_t kv_stride,
                 kvx_stream_t stream) {
  return guarded([&]() -> int {
    return store_call(pool, batch, nullptr, false, nullptr, 0, 0, nullptr, kv, kv_stride, (hipStream_t)stream);
  });
}

int store_latent_rope(kvx_latent_pool* pool, const kvx_batch* batch, const kvx_rope* rope, const void* q,
                      int32_t num_q_heads, int32_t q_dim, void* q_out, const void* kv, int64_t kv_stride,
                      kvx_stream_t stream) {
  return guarded([&]() -> int {
    return store_call(pool, batch, rope, true, q, num_q_heads, q_dim, q_out, kv, kv_stride, (hipStream_t)stream);
  });
}

int load_latent(kvx_latent_pool* pool, const kvx_batch* batch, void* out, int64_t out_stride, kvx_stream_t stream) {
  return guarded([&]() -> int {
    if (int rc = check_pool(pool)) return rc;
    std::vector<int64_t> qo;
    if (int rc = check_batch(batch, qo)) return rc;
    if (int rc = check_stride(out_stride, pool->latent_dim + kvx::kLatRope, "out_stride")) return rc;
    if (int rc = check_align(out, "out")) return rc;
    if (qo.back() == 0) return KVX_OK;
    if (!out) return report(KVX_EINVAL, "out is NULL");
    hipStream_t s = (hipStream_t)stream;
    OnDevice on;
    if (int rc = on.enter(pool->device)) return rc;
    if (int rc = check_stream(s, pool->device)) return rc;
    if (kvx::validate_mode())
      if (int rc = check_page_ids(pool->num_pages, batch, s)) return rc;
    kvx::LatentLoadParams p{};
    int64_t n_units = 0;
    if (int rc = place_units(pool, batch, qo, s, p, n_units)) return rc;
    p.pool = view(pool, batch);
    p.out = (uint16_t*)out;
    p.out_stride = out_stride;
    const hipError_t e = kvx::launch_load_latent(p, n_units, pool->latent_dim, pool->dtype == KVX_LATENT_FP8, s);
    if (e != hipSuccess) return hip_fail(e, "load_latent kernel launch");
    return p.units ? pool->st_rows.done(s) : KVX_OK;
  });
}

int latent_attention(kvx_latent_pool* pool, const kvx_batch* batch, const void* q, int32_t num_q_heads,
                     float sm_scale, void* out, float* lse, kvx_stream_t stream) {
  return guarded([&]() -> int {
    if (int rc = check_pool(pool)) return rc;
    std::vector<int64_t> qo;
    if (int rc = check_batch(batch, qo)) return rc;
    if (int rc = check_heads(batch, num_q_heads)) return rc;
    if (int rc = check_scale(sm_scale)) return rc;
    if (int rc = check_align(q, "q")) return rc;
    if (int rc = check_align(out, "out")) return rc;
    if (qo.back() == 0) return KVX_OK;
    if (!q || !out) return report(KVX_EINVAL, "q and out must be non-NULL");
    if (int rc = check_results(out, (size_t)pool->latent_dim * 2, lse, (size_t)qo.back() * num_q_heads, q,
                               (size_t)(pool->latent_dim + kvx::kLatRope) * 2))
      return rc;
    hipStream_t s = (hipStream_t)stream;
    OnDevice on;
    if (int rc = on.enter(pool->device)) return rc;
    if (int rc = check_stream(s, pool->device)) return rc;
    if (kvx::validate_mode())
      if (int rc = check_page_ids(pool->num_pages, batch, s)) return rc;
    std::vector<Member> members;
    for (int32_t r = 0; r < batch->num_reqs; r++)
      if (batch->extend_lens[r] > 0) members.push_back({r, qo[(size_t)r]});
    AbsorbedPlan plan;
    plan_absorbed(batch, members, num_q_heads, pool->latent_dim, pool->split_keys, plan);
    Blob blob;
    size_t units_at = 0, merges_at = 0;
    void* dev = nullptr;
    if (!plan.in_args) {
      units_at = blob.add(plan.units);
      merges_at = blob.add(plan.merges);
      if (int rc = pool->st_plan.upload(blob.bytes.data(), blob.bytes.size(), s, &dev)) return rc;
    }
    if (int rc = launch_absorbed(pool, batch, plan, (const uint8_t*)dev, units_at, merges_at, q, num_q_heads, sm_scale,
                                 out, lse, s))
      return rc;
    return plan.in_args ? KVX_OK : pool->st_plan.done(s);
  });
}

int latent_extend_attention(kvx_latent_pool* pool, const kvx_batch* batch, const kvx_latent_proj* proj,
                            const void* q, float sm_scale, void* out, float* lse, int32_t form,
                            kvx_stream_t stream) {
  return guarded([&]() -> int {
    if (int rc = check_pool(pool)) return rc;
    std::vector<int64_t> qo;
    if (int rc = check_batch(batch, qo)) return rc;
    if (proj == nullptr) return report(KVX_EINVAL, "proj is NULL");
    const int32_t Hq = proj->num_q_heads, D = proj->nope_dim, lat = pool->latent_dim;
    if (int rc = check_heads(batch, Hq)) return rc;
    if (D != 64 && D != 128) return report(KVX_EUNSUPPORTED, "nope_dim %d (supported: 64, 128)", D);
    if (proj->v_dim != D) return report(KVX_EUNSUPPORTED, "v_dim %d (supported: nope_dim = %d)", proj->v_dim, D);
    if (form != KVX_LATENT_AUTO && form != KVX_LATENT_ABSORBED && form != KVX_LATENT_EXPANDED)
      return report(KVX_EINVAL, "form %d", form);
    if (int rc = check_scale(sm_scale)) return rc;
    if (int rc = check_align(q, "q")) return rc;
    if (int rc = check_align(out, "out")) return rc;
    if (int rc = check_align(proj->w_uk, "w_uk")) return rc;
    if (int rc = check_align(proj->w_uv, "w_uv")) return rc;
    if (qo.back() == 0) return KVX_OK;
    if (!q || !out || !proj->w_uk || !proj->w_uv)
      return report(KVX_EINVAL, "q, out, w_uk and w_uv must be non-NULL");
    if (int rc = check_results(out, (size_t)D * 2, lse, (size_t)qo.back() * Hq, q, (size_t)(D + kvx::kLatRope) * 2,
                               proj->w_uk, proj->w_uv, (size_t)Hq * D * lat * 2))
      return rc;

    std::vector<bool> takes_absorbed((size_t)batch->num_reqs, form == KVX_LATENT_ABSORBED);
    if (form == KVX_LATENT_AUTO) takes_absorbed = choose_forms(batch, Hq, lat, D, pool->dtype == KVX_LATENT_FP8);
    std::vector<Member> absorbed;
    std::vector<int32_t> expanded;
    int64_t own_rows = 0;
    for (int32_t r = 0; r < batch->num_reqs; r++) {
      const int64_t E = batch->extend_lens[r];
      if (E == 0) continue;
      if (takes_absorbed[(size_t)r]) {
        absorbed.push_back({r, own_rows});
        own_rows += E;
      } else {
        expanded.push_back(r);
      }
    }
    const int64_t x_tokens = tokens_to_expand(batch, takes_absorbed);
    if (x_tokens > (int64_t)INT32_MAX)
      return report(KVX_EUNSUPPORTED, "%lld tokens to expand in one call", (long long)x_tokens);

    hipStream_t s = (hipStream_t)stream;
    OnDevice on;
    if (int rc = on.enter(pool->device)) return rc;
    if (int rc = check_stream(s, pool->device)) return rc;
    if (kvx::validate_mode())
      if (int rc = check_page_ids(pool->num_pages, batch, s)) return rc;

    // plans of everything, uploaded at once
    Blob blob;
    AbsorbedPlan ap;
    std::vector<LatentRows> rows;
    kvx::LatentProjParams ppar{};
    kvx::LatentExpandParams xpar{};
    kvx::LatentPrefillParams tpar[2] = {};
    kvx::LatentTileMergeParams mpar[2] = {};
    size_t a_units = 0, a_merges = 0, a_rows = 0;
    if (!absorbed.empty()) {
      plan_absorbed(batch, absorbed, Hq, lat, pool->split_keys, ap);
      for (size_t i = 0; i < absorbed.size();) {  // neighbours in the batch run on together
        size_t j = i;
        int64_t n = 0;
        const int64_t first = qo[(size_t)absorbed[i].req];
        while (j < absorbed.size() && qo[(size_t)absorbed[j].req] == first + n)
          n += batch->extend_lens[absorbed[j++].req];
        for (int64_t t = 0; t < n; t += kvx::kLatProjTok)
          rows.push_back({(int32_t)(first + t), (int32_t)(absorbed[i].row + t),
                          (int32_t)std::min<int64_t>(kvx::kLatProjTok, n - t), 0});
        i = j;
      }
      if (!ap.in_args) {
        a_units = blob.add(ap.units);
        a_merges = blob.add(ap.merges);
      }
      a_rows = place_list(rows, ppar.list, blob);
    }
    std::vector<LatentExpandUnit> x_units;
    std::vector<int64_t> x_row;
    int64_t x_rows = 0, per_head = 0;
    int32_t heads = Hq, last = Hq;
    ExpandedPlan xp, xl;  // of a group of heads, and of the last group where it is smaller
    size_t x_at = 0, t_at[2] = {}, m_at[2] = {};
    if (!expanded.empty()) {
      x_rows = expand_units(batch, expanded, x_units, x_row);
      per_head = 2 * x_rows * D * 2;
      heads = (int32_t)std::min<int64_t>(Hq, std::max<int64_t>(1, kMaxExpandBytes / per_head));
      heads = (int32_t)ceil_div(Hq, ceil_div(Hq, heads));
      last = Hq - heads * (int32_t)(ceil_div(Hq, heads) - 1);
      plan_expanded(batch, qo, expanded, x_row, heads, D, xp);
      x_at = place_list(x_units, xpar.list, blob);
      t_at[0] = place_list(xp.units, tpar[0].list, blob);
      m_at[0] = place_list(xp.merges, mpar[0].list, blob);
      if (last != heads) {
        plan_expanded(batch, qo, expanded, x_row, last, D, xl);
        t_at[1] = place_list(xl.units, tpar[1].list, blob);
        m_at[1] = place_list(xl.merges, mpar[1].list, blob);
      }
    }
    void* dev_v = nullptr;
    if (!blob.bytes.empty())
      if (int rc = pool->st_plan.upload(blob.bytes.data(), blob.bytes.size(), s, &dev_v)) return rc;
    const uint8_t* dev = (const uint8_t*)dev_v;

    if (!absorbed.empty()) {
      const size_t q_bytes = (size_t)own_rows * Hq * (lat + kvx::kLatRope) * 2, o_bytes = (size_t)own_rows * Hq * lat * 2;
      const size_t l_bytes = lse ? (size_t)own_rows * Hq * 4 : 0;
      if (int rc = pool->absorbed.ensure(q_bytes + o_bytes + l_bytes, s)) return rc;
      uint8_t* ws = (uint8_t*)pool->absorbed.ptr;
      float* own_lse = lse ? (float*)(ws + q_bytes + o_bytes) : nullptr;
      kvx::LatentProjParams& p = ppar;
      p.in = (const uint16_t*)q;
      p.w = (const uint16_t*)proj->w_uk;
      p.out = (uint16_t*)ws;
      p.rows = (const LatentRows*)(dev + a_rows);
      p.num_q_heads = Hq;
      hipError_t e = kvx::launch_latent_absorb(p, (int64_t)rows.size(), lat, D, s);
      if (e != hipSuccess) return hip_fail(e, "latent query product launch");
      if (int rc = launch_absorbed(pool, batch, ap, dev, a_units, a_merges, ws, Hq, sm_scale, ws + q_bytes, own_lse, s))
        return rc;
      p.in = (const uint16_t*)(ws + q_bytes);
      p.w = (const uint16_t*)proj->w_uv;
      p.out = (uint16_t*)out;
      p.lse_in = own_lse;
      p.lse_out = lse;
      e = kvx::launch_latent_output(p, (int64_t)rows.size(), lat, D, s);
      if (e != hipSuccess) return hip_fail(e, "latent output product launch");
      if (int rc = pool->absorbed.done(s)) return rc;
    }
    if (!expanded.empty()) {
      const size_t r_bytes = (size_t)x_rows * kvx::kLatRope * 2;
      if (int rc = pool->expanded.ensure(r_bytes + (size_t)per_head * heads, s)) return rc;
      const int64_t n_parts = std::max(xp.n_parts, xl.n_parts);
      const size_t per_part = (size_t)kvx::kLatTileTok * D;
      if (n_parts > 0)
        if (int rc = pool->parts.ensure((size_t)n_parts * (per_part + kvx::kLatTileTok) * sizeof(float), s)) return rc;
      uint8_t* ws = (uint8_t*)pool->expanded.ptr;
      for (int32_t h0 = 0; h0 < Hq; h0 += heads) {
        const int32_t n = std::min(heads, Hq - h0);
        const bool tail = n != heads;
        const ExpandedPlan& plan = tail ? xl : xp;
        kvx::LatentExpandParams& x = xpar;
        x.pool = view(pool, batch);
        x.w_uk = (const uint16_t*)proj->w_uk + (size_t)h0 * D * lat;
        x.w_uv = (const uint16_t*)proj->w_uv + (size_t)h0 * D * lat;
        x.kx = (uint16_t*)(ws + r_bytes);
        x.vx = x.kx + (size_t)n * x_rows * D;
        x.rx = h0 == 0 ? (uint16_t*)ws : nullptr;
        x.units = (const LatentExpandUnit*)(dev + x_at);
        x.x_rows = x_rows;
        x.heads = n;
        hipError_t e = kvx::launch_latent_expand(x, (int64_t)x_units.size(), lat, D, pool->dtype == KVX_LATENT_FP8, s);
        if (e != hipSuccess) return hip_fail(e, "latent expansion launch");
        kvx::LatentPrefillParams& p = tpar[tail];
        p.q = (const uint16_t*)q;
        p.out = (uint16_t*)out;
        p.lse = lse;
        p.kx = x.kx;
        p.vx = x.vx;
        p.rx = (const uint16_t*)ws;
        p.units = (const LatentTile*)(dev + t_at[tail]);
        p.o_part = (float*)pool->parts.ptr;
        p.lse_part = n_parts ? p.o_part + (size_t)plan.n_parts * per_part : nullptr;
        p.x_rows = x_rows;
        p.num_q_heads = Hq;
        p.head0 = h0;
        p.scale_log2 = sm_scale * kLog2e;
        e = kvx::launch_latent_prefill(p, (int64_t)plan.units.size(), D, s);
        if (e != hipSuccess) return hip_fail(e, "expanded attention launch");
        if (!plan.merges.empty()) {
          kvx::LatentTileMergeParams& m = mpar[tail];
          m.merges = (const LatentTileMerge*)(dev + m_at[tail]);
          m.o_part = p.o_part;
          m.lse_part = p.lse_part;
          m.out = p.out;
          m.lse = lse;
          m.num_q_heads = Hq;
          m.head0 = h0;
          e = kvx::launch_latent_tile_merge(m, (int64_t)plan.merges.size(), D, s);
          if (e != hipSuccess) return hip_fail(e, "expanded merge launch");
        }
      }
      if (int rc = pool->expanded.done(s)) return rc;
      if (n_parts > 0)
        if (int rc = pool->parts.done(s)) return rc;
    }
    return blob.bytes.empty() ? KVX_OK : pool->st_plan.done(s);
  });
}

}  // extern "C"
