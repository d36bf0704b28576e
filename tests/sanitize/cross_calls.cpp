// Checks of the host code of cross_attention and load_kv (csrc/kvx_host.cpp, csrc/kvx_load.cpp) over
// a stand-in for the HIP runtime with two devices: what is refused, that the units of a call
// cover every (query, key) pair once, and what a call does with devices.  Built by
// tests/test_cross_host.py with the sanitizers; kernels are not launched, their units are read.
// The argument names the check.

#include "kvx_host.cpp"
#include "kvx_load.cpp"

#include <map>
#include <new>
#include <random>
#include <tuple>

// Host allocations until one fails; < 0: none does.
static int g_allocs = -1;
void* operator new(size_t n) {
  if (g_allocs >= 0 && g_allocs-- == 0) throw std::bad_alloc();
  if (void* p = std::malloc(n)) return p;
  throw std::bad_alloc();
}
void* operator new(size_t n, const std::nothrow_t&) noexcept { return std::malloc(n); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

struct ihipStream_t {
  int device;
  bool capturing;
};

namespace fake {
int current = 0;
}

extern "C" {
hipError_t hipGetDevice(int* d) { return *d = fake::current, hipSuccess; }
hipError_t hipSetDevice(int d) { return fake::current = d, hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "stand-in error"; }
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* st) {
  *st = s != nullptr && s->capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipStreamGetDevice(hipStream_t s, hipDevice_t* d) { return *d = s->device, hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return *e = (hipEvent_t)std::malloc(1), hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t e) { return std::free((void*)e), hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipHostMalloc(void** p, size_t n, unsigned) { return *p = std::malloc(n), hipSuccess; }
hipError_t hipHostFree(void* p) { return std::free(p), hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { return *p = std::malloc(n), hipSuccess; }
hipError_t hipFree(void* p) { return std::free(p), hipSuccess; }
hipError_t hipMallocAsync(void** p, size_t n, hipStream_t) {
  return *p = std::malloc(n < (1 << 22) ? n : 64), hipSuccess;  // partial results are never touched here
}
hipError_t hipFreeAsync(void* p, hipStream_t) { return std::free(p), hipSuccess; }
hipError_t hipMemset(void* p, int v, size_t n) { return std::memset(p, v, n), hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { return std::memcpy(d, s, n), hipSuccess; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) {
  return std::memcpy(d, s, n), hipSuccess;
}
hipError_t hipPointerGetAttributes(hipPointerAttribute_t*, const void*) { return hipErrorInvalidValue; }
}

#define CHECK(cond)                                                                                        \
  do {                                                                                                     \
    if (!(cond)) {                                                                                         \
      std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #cond, kvx_last_error());       \
      std::exit(3);                                                                                        \
    }                                                                                                      \
  } while (0)

// What the launches of a call compute: for every row (token, head of the KV heads) its key ranges.
struct Range {
  int32_t page_base, begin, end, part;
};
static std::map<std::pair<int64_t, int32_t>, std::vector<Range>> g_tiled, g_stepped;
static std::map<std::pair<int64_t, int32_t>, std::pair<int32_t, int32_t>> g_tile_merge, g_step_merge;  // part0, parts
static std::map<std::pair<int64_t, int32_t>, int> g_empty;
static std::map<int64_t, int32_t> g_sees;  // keys that a token of a draft sees
static int g_launches = 0, g_on = -1, g_loads = 0, g_causal = 0;

static void forget() {
  g_tiled.clear();
  g_stepped.clear();
  g_tile_merge.clear();
  g_step_merge.clear();
  g_empty.clear();
  g_sees.clear();
  g_launches = g_loads = 0;
}

namespace kvx {
hipError_t launch_extend_attention(const AttnParams& p, int64_t n, int, bool, bool, hipStream_t) {
  g_launches++;
  g_on = fake::current;
  CHECK(p.cross == 1 && p.mixed == 0);
  for (int64_t i = 0; i < n; i++) {
    const AttnUnit u = p.compact ? unit_from_plan(*p.compact, (const uint32_t*)p.compact->words, (int)i) : p.units[i];
    if (u.key_end <= u.key_begin) continue;
    const int head = u.head_ntok >> 16, ntok = u.head_ntok & 0xFFFF;
    CHECK(ntok >= 1 && ntok <= p.tile_tok && head < p.num_kv_heads);
    CHECK(u.key_end <= u.q_pos0 + 1 && u.key_begin % kTileKeys == 0 && u.key_begin <= u.q_pos0);
    for (int t = 0; t < ntok; t++)
      g_tiled[{u.qo_row0 + t, head}].push_back(Range{u.page_base, u.key_begin, u.key_end, u.part});
  }
  return hipSuccess;
}
hipError_t launch_merge(const MergeParams& p, int64_t n, int, hipStream_t) {
  for (int64_t i = 0; i < n; i++) {
    MergeUnit m;
    if (p.plan.n > 0) {
      m = p.plan.merge[i / p.plan.heads];
      m.head_ntok += (int32_t)(i % p.plan.heads) << 16;
      m.part0 += (int32_t)(i % p.plan.heads) * m.nparts;
    } else {
      m = p.merges[i];
    }
    for (int t = 0; t < (m.head_ntok & 0xFFFF); t++) {
      CHECK(!g_tile_merge.count({m.qo_row0 + t, m.head_ntok >> 16}));
      g_tile_merge[{m.qo_row0 + t, m.head_ntok >> 16}] = {m.part0, m.nparts};
    }
  }
  return hipSuccess;
}
hipError_t launch_decode(const DecodeParams& dp, int64_t, int, bool, hipStream_t) {
  g_launches++;
  g_on = fake::current;
  CHECK(dp.rows != nullptr);
  const RowsParams& p = *dp.rows;
  CHECK(p.causal == g_causal && (p.blocks == 1 || p.blocks == 2));
  const uint32_t* w = p.words ? p.words : p.in_args;
  if (!p.words) CHECK(p.n_entries * kRowsEntryWords + p.n_codes <= kRowsWords);
  bool parts = false;
  for (int32_t i = 0; i < p.n_codes; i++) {
    const uint32_t code = w[kRowsEntryWords * p.n_entries + i];
    CHECK((int32_t)(code >> kRowsRangeBits) < p.n_entries);
    RowsEntry e;
    std::memcpy(&e, w + kRowsEntryWords * (code >> kRowsRangeBits), sizeof e);
    const int32_t range = (int32_t)(code & ((1u << kRowsRangeBits) - 1));
    CHECK(e.ntok >= 1 && e.len > 0 && e.len % kDecodeChunkAlign == 0);
    const int32_t n = e.keys > 0 ? (e.keys - 1) / e.len + 1 : 1;
    CHECK(range < n && (e.part0 >= 0) == (n > 1));
    if (e.keys > 0) CHECK(e.ntok * p.group <= 16 * p.blocks);
    parts |= n > 1;
    for (int32_t h = 0; h < p.num_kv_heads; h++)
      for (int t = 0; t < e.ntok; t++) {
        const std::pair<int64_t, int32_t> at{e.qo_row + t, h};
        if (p.causal) g_sees[e.qo_row + t] = e.keys - (e.ntok - 1 - t);
        if (e.keys == 0) {
          g_empty[at]++;
          continue;
        }
        const int64_t begin = (int64_t)range * e.len, end = std::min<int64_t>(e.keys, begin + e.len);
        g_stepped[at].push_back(Range{e.page_base, (int32_t)begin, (int32_t)end, n > 1 ? e.part0 + h * n + range : -1});
        if (n > 1) g_step_merge[at] = {e.part0 + h * n, n};
      }
  }
  CHECK(parts == (p.any_parts != 0));
  return hipSuccess;
}
hipError_t launch_decode_merge(const DecodeMergeParams&, int64_t, int, hipStream_t) { std::exit(4); }
hipError_t launch_store_kv(const StoreParams&, int64_t, int, bool, hipStream_t) { std::exit(4); }
hipError_t launch_store_kv_rope(const RopeParams&, int64_t, int, bool, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_page_move(const PageMoveParams&, int64_t, hipStream_t) { std::exit(4); }
hipError_t launch_page_io(const PageIoParams&, int64_t, int, int, hipStream_t) { std::exit(4); }
hipError_t launch_load_kv(const LoadParams&, int64_t, int, int32_t, hipStream_t) {
  g_loads++;
  g_on = fake::current;
  return hipSuccess;
}
}  // namespace kvx

namespace {

struct TestBatch {
  std::vector<int32_t> P, E, indptr{0}, ids;
  kvx_batch b{};
  TestBatch(std::vector<int32_t> p, std::vector<int32_t> e, int extra = 0) : P(std::move(p)), E(std::move(e)) {
    for (size_t r = 0; r < P.size(); r++) indptr.push_back(indptr.back() + (P[r] + 15) / 16 + extra);
    ids.resize((size_t)std::max(1, indptr.back()));
    b = kvx_batch{(int32_t)P.size(), P.data(), E.data(), indptr.data(), ids.data()};
  }
  int64_t total() const {
    int64_t t = 0;
    for (const int32_t e : E) t += e;
    return t;
  }
};

alignas(16) uint8_t g_mem[64];
// Addresses that are never touched, far enough apart for any call here.
void* far_away(int i) { return (void*)((uintptr_t)(i + 1) << 40); }

kvx_pool pool_of(int32_t hkv, int32_t d, int32_t dtype, int device = 0) {
  kvx_pool p;
  p.num_pages = 1 << 20;
  p.num_kv_heads = hkv;
  p.head_dim = d;
  p.kv_dtype = dtype;
  p.elem_bytes = dtype == KVX_KV_BF16 ? 2 : 1;
  p.device = device;
  return p;
}

void release(kvx_pool& p) {
  p.st_load.release();
  p.st_attn.release();
  p.parts.release();
}

int cross(kvx_pool& p, const TestBatch& t, int32_t hq, hipStream_t s = nullptr) {
  forget();
  return cross_attention(&p, &t.b, far_away(1), hq, 0.125f, far_away(2), nullptr, s);
}

// Every row has its request's keys once; parts are of its merge, all of them, or it has none.
void check_rows(const kvx_pool& p, const TestBatch& t) {
  int64_t row = 0;
  for (size_t r = 0; r < t.P.size(); r++)
    for (int32_t e = 0; e < t.E[r]; e++, row++)
      for (int32_t h = 0; h < p.num_kv_heads; h++) {
        const std::pair<int64_t, int32_t> at{row, h};
        CHECK((int)g_tiled.count(at) + (int)g_stepped.count(at) + (int)g_empty.count(at) == 1);
        if (t.P[r] == 0) {
          CHECK(g_empty[at] == 1);
          continue;
        }
        const bool tiled = g_tiled.count(at) != 0;
        std::vector<Range> ranges = tiled ? g_tiled[at] : g_stepped[at];
        std::sort(ranges.begin(), ranges.end(), [](const Range& x, const Range& y) { return x.begin < y.begin; });
        int32_t upto = 0;
        for (const Range& x : ranges) {
          CHECK(x.begin == upto && x.end > x.begin && x.page_base == t.indptr[r]);
          upto = x.end;
        }
        CHECK(upto == t.P[r]);
        auto& merges = tiled ? g_tile_merge : g_step_merge;
        if (ranges.size() == 1 && ranges[0].part < 0) {
          CHECK(!merges.count(at));
          continue;
        }
        CHECK(merges.count(at) && merges[at].second == (int32_t)ranges.size());
        std::vector<int32_t> parts;
        for (const Range& x : ranges) parts.push_back(x.part - merges[at].first);
        std::sort(parts.begin(), parts.end());
        for (size_t i = 0; i < parts.size(); i++) CHECK(parts[i] == (int32_t)i);
      }
  const int64_t rows = t.total() * p.num_kv_heads;
  CHECK((int64_t)(g_tiled.size() + g_stepped.size() + g_empty.size()) == rows);
}

void coverage() {
  std::mt19937 rng(7);
  auto log_uniform = [&](double hi) { return (int32_t)std::exp(std::uniform_real_distribution<double>(0, std::log(hi))(rng)); };
  for (int trial = 0; trial < 400; trial++) {
    const int n = 1 + (int)(rng() % (trial % 10 == 0 ? 300 : 12));
    std::vector<int32_t> P, E;
    for (int r = 0; r < n; r++) {
      P.push_back(rng() % 8 == 0 ? 0 : log_uniform(trial % 3 == 0 ? 20000 : 900));
      E.push_back(rng() % 8 == 0 ? 0 : log_uniform(trial % 2 == 0 ? 12 : 600));
    }
    const int32_t hkv = 1 + (int32_t)(rng() % 10);
    const int32_t groups[] = {1, 2, 3, 4, 5, 7, 8, 12, 16, 17, 20, 100};
    const int32_t g = groups[rng() % 12];
    kvx_pool p = pool_of(hkv, rng() % 2 ? 64 : 128, (int32_t)(rng() % 3));
    if (trial % 4 == 0) p.split_keys = 64 * (1 + (int32_t)(rng() % 8));
    const TestBatch t(P, E, (int)(rng() % 2));
    CHECK(cross(p, t, hkv * g) == KVX_OK);
    check_rows(p, t);
    release(p);
  }
  // requests without tokens, many queries among them, and nothing else; more of them than arguments hold
  kvx_pool p = pool_of(3, 64, KVX_KV_BF16);
  for (const auto& t : {TestBatch({0}, {5000}), TestBatch({0, 0, 0}, {1, 0, 40}), TestBatch(std::vector<int32_t>(500, 0), std::vector<int32_t>(500, 3))}) {
    CHECK(cross(p, t, 60) == KVX_OK);
    check_rows(p, t);
  }
  CHECK(cross(p, TestBatch({}, {}), 6) == KVX_OK && g_launches == 0);
  CHECK(cross(p, TestBatch({33, 0}, {0, 0}), 6) == KVX_OK && g_launches == 0);
  release(p);
}

// extend_attention of few tokens a request on a page-scaled pool: the same launches, each token
// seeing one key more than the one before it.
void drafts() {
  std::mt19937 rng(11);
  for (int trial = 0; trial < 300; trial++) {
    const int32_t groups[] = {1, 2, 3, 5, 8, 16, 20, 32};
    const int32_t hkv = 1 + (int32_t)(rng() % 8), g = groups[rng() % 8];
    std::vector<int32_t> P, E, total;
    for (int r = 0, n = 1 + (int)(rng() % (trial % 10 == 0 ? 250 : 10)); r < n; r++) {
      P.push_back((int32_t)(rng() % 3000));
      E.push_back((int32_t)(rng() % (4 * (32 / g) + 1)));
      total.push_back(P.back() + E.back());
    }
    TestBatch t(total, E);  // pages for prefix and suffix
    t.b.prefix_lens = P.data();
    kvx_pool p = pool_of(hkv, rng() % 2 ? 64 : 128, KVX_KV_FP8_PAGE);
    if (trial % 4 == 0) p.split_keys = 64 * (1 + (int32_t)(rng() % 8));
    forget();
    g_causal = 1;
    CHECK(extend_attention(&p, &t.b, far_away(1), hkv * g, 0.125f, far_away(2), nullptr, nullptr) == KVX_OK);
    g_causal = 0;
    CHECK(g_tiled.empty() && g_launches == (t.total() > 0 ? 1 : 0));
    int64_t row = 0;
    for (size_t r = 0; r < P.size(); r++)
      for (int32_t e = 0; e < E[r]; e++, row++) {
        CHECK(g_sees[row] == P[r] + e + 1);
        for (int32_t h = 0; h < hkv; h++) {
          std::vector<Range> ranges = g_stepped[{row, h}];
          std::sort(ranges.begin(), ranges.end(), [](const Range& x, const Range& y) { return x.begin < y.begin; });
          int32_t upto = 0;
          for (const Range& x : ranges) {
            CHECK(x.begin == upto && x.page_base == t.indptr[r]);
            upto = x.end;
          }
          CHECK(upto >= P[r] + e + 1 && upto <= P[r] + E[r]);
        }
      }
    CHECK((int64_t)g_sees.size() == t.total());
    release(p);
  }
}

// Launches that a grid cannot hold are refused before any work.
void limits() {
  kvx_pool p = pool_of(32, 64, KVX_KV_BF16);
  const TestBatch many(std::vector<int32_t>(600000, 1), std::vector<int32_t>(600000, 1));
  CHECK(cross(p, many, 32) == KVX_EUNSUPPORTED && g_launches == 0);
  release(p);
  p = pool_of(1, 64, KVX_KV_BF16);
  const TestBatch more(std::vector<int32_t>(1 << 20, 1), std::vector<int32_t>(1 << 20, 1));
  CHECK(cross(p, more, 1) == KVX_EUNSUPPORTED && g_launches == 0);
  TestBatch longest({300000000}, {300000000});
  std::vector<int32_t> zero{0};
  longest.b.prefix_lens = zero.data();
  CHECK(load_kv(&p, &longest.b, far_away(1), far_away(2), nullptr) == KVX_EUNSUPPORTED && g_loads == 0);
  release(p);
  p = pool_of(1, 64, KVX_KV_FP8_PAGE);
  CHECK(store_kv(&p, &longest.b, far_away(1), far_away(2), nullptr) == KVX_EUNSUPPORTED);
  release(p);
}

void refusals() {
  kvx_pool p = pool_of(2, 64, KVX_KV_BF16);
  const TestBatch t({40, 0, 7}, {3, 2, 1});
  void *q = far_away(1), *out = far_away(2);
  float* lse = (float*)far_away(3);
  auto call = [&](kvx_pool* pool, const kvx_batch* b, const void* q_, int32_t hq, float scale, void* out_, float* lse_) {
    forget();
    const int rc = cross_attention(pool, b, q_, hq, scale, out_, lse_, nullptr);
    CHECK(rc == KVX_OK || (g_launches == 0 && kvx_last_error()[0] != 0));
    return rc;
  };
  CHECK(call(&p, &t.b, q, 6, 0.125f, out, lse) == KVX_OK);
  CHECK(call(nullptr, &t.b, q, 6, 0.125f, out, lse) == KVX_EINVAL);
  CHECK(call(&p, nullptr, q, 6, 0.125f, out, lse) == KVX_EINVAL);
  for (const int32_t hq : {0, -2, 3}) CHECK(call(&p, &t.b, q, hq, 0.125f, out, lse) == KVX_EINVAL);
  CHECK(call(&p, &t.b, q, 2 * 257, 0.125f, out, lse) == KVX_EUNSUPPORTED);
  for (const float s : {0.0f, -1.0f, (float)INFINITY, (float)NAN}) CHECK(call(&p, &t.b, q, 6, s, out, lse) == KVX_EINVAL);
  CHECK(call(&p, &t.b, nullptr, 6, 0.125f, out, lse) == KVX_EINVAL);
  CHECK(call(&p, &t.b, q, 6, 0.125f, nullptr, lse) == KVX_EINVAL);
  CHECK(call(&p, &t.b, (char*)q + 8, 6, 0.125f, out, lse) == KVX_EINVAL);
  CHECK(call(&p, &t.b, q, 6, 0.125f, (char*)out + 2, lse) == KVX_EINVAL);
  CHECK(call(&p, &t.b, q, 6, 0.125f, out, (float*)((char*)lse + 2)) == KVX_EINVAL);
  CHECK(call(&p, &t.b, q, 6, 0.125f, (char*)q + 6 * 6 * 64 * 2 - 16, lse) == KVX_EINVAL);  // the last 16 bytes
  CHECK(call(&p, &t.b, q, 6, 0.125f, (char*)q + 6 * 6 * 64 * 2, lse) == KVX_OK);
  CHECK(call(&p, &t.b, q, 6, 0.125f, q, lse) == KVX_EINVAL);
  CHECK(call(&p, &t.b, q, 6, 0.125f, out, (float*)q) == KVX_EINVAL);
  CHECK(call(&p, &t.b, q, 6, 0.125f, out, (float*)out + 5) == KVX_EINVAL);
  TestBatch bad = t;
  auto with = [&](auto change) {
    bad = TestBatch({40, 0, 7}, {3, 2, 1});
    change(bad);
    return call(&p, &bad.b, q, 6, 0.125f, out, lse);
  };
  CHECK(with([](TestBatch& x) { x.P[0] = -1; }) == KVX_EINVAL);
  CHECK(with([](TestBatch& x) { x.E[1] = -1; }) == KVX_EINVAL);
  CHECK(with([](TestBatch& x) { x.P[0] = 49; }) == KVX_EINVAL);  // four pages for three listed
  CHECK(with([](TestBatch& x) { x.P[0] = 48; }) == KVX_OK);
  CHECK(with([](TestBatch& x) { x.E[2] = 1000; }) == KVX_OK);    // queries need no pages
  CHECK(with([](TestBatch& x) { x.indptr[0] = 1; }) == KVX_EINVAL);
  CHECK(with([](TestBatch& x) { x.b.page_ids = nullptr; }) == KVX_EINVAL);
  CHECK(with([](TestBatch& x) { x.b.prefix_lens = nullptr; }) == KVX_EINVAL);
  CHECK(with([](TestBatch& x) { x.b.num_reqs = -1; }) == KVX_EINVAL);
  CHECK(with([](TestBatch& x) { x.E[0] = x.E[1] = INT32_MAX - 2000; }) == KVX_EINVAL);  // too many rows
  release(p);

  p = pool_of(2, 64, KVX_KV_FP8_PAGE);
  auto load = [&](kvx_pool* pool, const kvx_batch* b, void* k, void* v) {
    forget();
    const int rc = load_kv(pool, b, k, v, nullptr);
    CHECK(rc == KVX_OK || (g_loads == 0 && kvx_last_error()[0] != 0));
    return rc;
  };
  const TestBatch u({16, 4}, {0, 0}, 1);
  TestBatch rows({16, 4}, {16, 12}, 2);
  CHECK(load(&p, &rows.b, q, out) == KVX_OK && g_loads == 1);
  CHECK(load(&p, &u.b, q, out) == KVX_OK && g_loads == 0);
  CHECK(load(nullptr, &rows.b, q, out) == KVX_EINVAL);
  CHECK(load(&p, nullptr, q, out) == KVX_EINVAL);
  CHECK(load(&p, &rows.b, nullptr, out) == KVX_EINVAL);
  CHECK(load(&p, &rows.b, q, nullptr) == KVX_EINVAL);
  CHECK(load(&p, &rows.b, (char*)q + 4, out) == KVX_EINVAL);
  CHECK(load(&p, &rows.b, q, (char*)out + 4) == KVX_EINVAL);
  CHECK(load(&p, &rows.b, q, (char*)q + 28 * 2 * 64 * 2 - 16) == KVX_EINVAL);
  CHECK(load(&p, &rows.b, q, (char*)q + 28 * 2 * 64 * 2) == KVX_OK);
  rows.E[0] = 100;  // past its pages
  CHECK(load(&p, &rows.b, q, out) == KVX_EINVAL);
  release(p);
}

void streams() {
  kvx_pool p = pool_of(2, 64, KVX_KV_BF16, 1);
  const TestBatch t({40, 0, 700}, {3, 2, 90}, 6);
  ihipStream_t of0{0, false}, of1{1, false}, captured{1, true};
  for (const int before : {0, 1}) {
    fake::current = before;
    CHECK(cross(p, t, 6) == KVX_OK && g_on == 1 && fake::current == before && g_launches == 2);
    CHECK(cross(p, t, 6, &of1) == KVX_OK && g_on == 1 && fake::current == before);
    CHECK(cross(p, t, 6, &of0) == KVX_EINVAL && g_launches == 0 && fake::current == before);
    CHECK(cross(p, t, 6, &captured) == KVX_EUNSUPPORTED && g_launches == 0 && fake::current == before);
    forget();
    CHECK(load_kv(&p, &t.b, far_away(1), far_away(2), &of1) == KVX_OK && g_loads == 1 && fake::current == before);
    CHECK(load_kv(&p, &t.b, far_away(1), far_away(2), &of0) == KVX_EINVAL && g_loads == 1);
    CHECK(load_kv(&p, &t.b, far_away(1), far_away(2), &captured) == KVX_EUNSUPPORTED && g_loads == 1);
  }
  fake::current = 0;
  release(p);
}

// Whichever host allocation of a call fails, the call says so and leaves the pool as it was.
void memory() {
  std::vector<int32_t> P, E;
  for (int i = 0; i < 300; i++) {
    P.push_back(1 + 97 * i);
    E.push_back(1 + i % 3);
  }
  const TestBatch large(P, E, 1), small({700, 900}, {1, 2}, 1), tiles({700, 900}, {400, 3}, 25);
  kvx_rope rope{10000.0, nullptr, 64, KVX_ROPE_HALF, nullptr, nullptr, 1e-6f};
  kvx_pool p = pool_of(2, 64, KVX_KV_FP8_PAGE);
  for (const TestBatch* t : {&large, &small, &tiles})
    for (int what = 0; what < 5; what++) {
      if (what == 0 && t == &tiles) continue;  // the stand-in's tiles are cross attention's
      g_causal = what == 0;
      auto call = [&]() {
        if (what == 0) return extend_attention(&p, &t->b, far_away(1), 6, 0.1f, far_away(2), nullptr, nullptr);
        if (what == 1) return cross_attention(&p, &t->b, far_away(1), 6, 0.1f, far_away(2), nullptr, nullptr);
        if (what == 2) return store_kv(&p, &t->b, far_away(1), far_away(2), nullptr);
        if (what == 3) return store_kv_rope(&p, &t->b, &rope, nullptr, 0, nullptr, far_away(1), far_away(2), nullptr);
        return load_kv(&p, &t->b, far_away(1), far_away(2), nullptr);
      };
      int failed = 0, rc = KVX_ENOMEM;
      for (; rc == KVX_ENOMEM && failed < 10000; failed++) {
        forget();
        g_allocs = failed;
        rc = call();
        const bool whole = g_allocs >= 0;
        g_allocs = -1;
        CHECK(rc == (whole ? KVX_OK : KVX_ENOMEM));
      }
      CHECK(rc == KVX_OK && failed > 1);
    }
  g_causal = 0;
  p.st_store.release();
  release(p);
}

// A pool's own refusals, and what a page-scaled pool adds to its buffers.
void pools() {
  kvx_pool* p = nullptr;
  const float one[2] = {1.0f, 1.0f};
  CHECK(kv_pool_create(4, 16, 2, 64, KVX_KV_FP8_PAGE, one, one, &p) == KVX_EINVAL && p == nullptr);
  CHECK(kv_pool_create(4, 16, 2, 64, KVX_KV_FP8_PAGE, nullptr, one, &p) == KVX_EINVAL && p == nullptr);
  CHECK(kv_pool_create(4, 16, 2, 64, 3, nullptr, nullptr, &p) == KVX_EINVAL && p == nullptr);
  for (const int32_t heads : {1, 2, 5}) {
    CHECK(kv_pool_create(4, 16, heads, 64, KVX_KV_FP8_PAGE, nullptr, nullptr, &p) == KVX_OK);
    int64_t bytes = 0;
    CHECK(kv_pool_record_bytes(p, &bytes) == KVX_OK);
    CHECK(bytes % 16 == 0 && bytes - 2 * heads * 16 * 64 >= 8 * heads && bytes - 2 * heads * 16 * 64 < 8 * heads + 16);
    kvx_pool_layout lay;
    CHECK(kv_pool_layout(p, &lay) == KVX_OK && lay.elem_bytes == 1 && lay.kv_dtype == KVX_KV_FP8_PAGE);
    CHECK(lay.k_scale != nullptr && lay.v_scale == lay.k_scale + 1);
    CHECK(kv_pool_set_scaled_q(p, 1) == KVX_OK);
    CHECK(kv_pool_destroy(p) == KVX_OK);
  }
}

}  // namespace

int main(int argc, char** argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  (void)g_mem;
  if (what == "coverage") coverage();
  else if (what == "drafts") drafts();
  else if (what == "limits") limits();
  else if (what == "refusals") refusals();
  else if (what == "streams") streams();
  else if (what == "pools") pools();
  else if (what == "memory") memory();
  else return 2;
  std::printf("%s passed\n", what.c_str());
  return 0;
}
