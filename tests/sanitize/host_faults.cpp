// Checks of the KV pool's host code (csrc/kvx_host.cpp, csrc/kvx_load.cpp) over a stand-in for the HIP
// runtime: host memory that stays short, and the plans of batches of few rows.  Built by
// tests/test_host_faults.py with the sanitizers; kernels are not launched.  The argument names the
// check.

#include "kvx_host.cpp"
#include "kvx_load.cpp"

#include <cmath>
#include <functional>
#include <new>
#include <string>

// Host allocations until memory is short, from when on each one fails; < 0: it never is.
static int g_left = -1;
static bool short_of_memory() {
  if (g_left < 0) return false;
  if (g_left == 0) return true;
  g_left--;
  return false;
}
void* operator new(size_t n) {
  if (!short_of_memory())
    if (void* p = std::malloc(n)) return p;
  throw std::bad_alloc();
}
void* operator new(size_t n, const std::nothrow_t&) noexcept { return short_of_memory() ? nullptr : std::malloc(n); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

static int g_device_blocks = 0;
static void* device_block(size_t n) {
  g_device_blocks++;
  return std::malloc(n < (1 << 22) ? n : 64);  // partial results are never touched here
}

extern "C" {
hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "stand-in error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* st) {
  return *st = hipStreamCaptureStatusNone, hipSuccess;
}
hipError_t hipStreamGetDevice(hipStream_t, hipDevice_t* d) { return *d = 0, hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return *e = (hipEvent_t)std::malloc(1), hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t e) { return std::free((void*)e), hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipHostMalloc(void** p, size_t n, unsigned) { return *p = std::malloc(n), hipSuccess; }
hipError_t hipHostFree(void* p) { return std::free(p), hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { return *p = device_block(n), hipSuccess; }
hipError_t hipFree(void* p) { return g_device_blocks--, std::free(p), hipSuccess; }
hipError_t hipMallocAsync(void** p, size_t n, hipStream_t) { return *p = device_block(n), hipSuccess; }
hipError_t hipFreeAsync(void* p, hipStream_t) { return g_device_blocks--, std::free(p), hipSuccess; }
hipError_t hipMemset(void* p, int v, size_t n) { return std::memset(p, v, n), hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { return std::memcpy(d, s, n), hipSuccess; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) {
  return std::memcpy(d, s, n), hipSuccess;
}
hipError_t hipPointerGetAttributes(hipPointerAttribute_t* a, const void* p) {
  a->type = hipMemoryTypeHost;
  a->hostPointer = a->devicePointer = const_cast<void*>(p);
  return hipSuccess;
}
}

#define CHECK(cond)                                                                                        \
  do {                                                                                                     \
    if (!(cond)) {                                                                                         \
      std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #cond, kvx_last_error());       \
      std::exit(3);                                                                                        \
    }                                                                                                      \
  } while (0)

static int g_launches = 0;

namespace kvx {
hipError_t launch_extend_attention(const AttnParams&, int64_t, int, bool, bool, hipStream_t) { return g_launches++, hipSuccess; }
hipError_t launch_merge(const MergeParams&, int64_t, int, hipStream_t) { return hipSuccess; }
hipError_t launch_decode(const DecodeParams&, int64_t, int, bool, hipStream_t) { return g_launches++, hipSuccess; }
hipError_t launch_decode_merge(const DecodeMergeParams&, int64_t, int, hipStream_t) { return hipSuccess; }
hipError_t launch_store_kv(const StoreParams&, int64_t, int, bool, hipStream_t) { return g_launches++, hipSuccess; }
hipError_t launch_store_kv_rope(const RopeParams&, int64_t, int, bool, bool, hipStream_t) { return g_launches++, hipSuccess; }
hipError_t launch_page_move(const PageMoveParams&, int64_t, hipStream_t) { return g_launches++, hipSuccess; }
hipError_t launch_page_io(const PageIoParams&, int64_t, int, int, hipStream_t) { return g_launches++, hipSuccess; }
hipError_t launch_load_kv(const LoadParams&, int64_t, int, int32_t, hipStream_t) { return g_launches++, hipSuccess; }
}  // namespace kvx

namespace {

struct TestBatch {
  std::vector<int32_t> P, E, indptr{0}, ids;
  kvx_batch b{};
  TestBatch(std::vector<int32_t> p, std::vector<int32_t> e) : P(std::move(p)), E(std::move(e)) {
    for (size_t r = 0; r < P.size(); r++) indptr.push_back(indptr.back() + (P[r] + E[r] + 15) / 16);
    ids.resize((size_t)std::max(1, indptr.back()));
    b = kvx_batch{(int32_t)P.size(), P.data(), E.data(), indptr.data(), ids.data()};
  }
};

// Addresses that are never touched, far enough apart for any call here.
void* far_away(int i) { return (void*)((uintptr_t)(i + 1) << 40); }

uint8_t g_arena[KVX_NOALLOC_PLAN_BYTES];  // the partial results behind it are never touched here
int arena(int, void** p) { return *p = g_arena, KVX_OK; }

// With memory short from any allocation on, a call says so, with a message, queues nothing, keeps nothing
// and lets no exception out; with enough of it, it succeeds.
void memory() {
  std::vector<int32_t> P, E;
  for (int i = 0; i < 300; i++) {
    P.push_back(1 + 97 * i);
    E.push_back(1 + i % 3);
  }
  const TestBatch large(P, E), ones(P, std::vector<int32_t>(P.size(), 1)), tiles({700, 900}, {400, 333}), mixed({700, 90, 3}, {1, 400, 1});
  kvx_rope rope{10000.0, nullptr, 64, KVX_ROPE_HALF, nullptr, nullptr, 1e-6f};
  const kvx::FixedScratch fixed{KVX_NOALLOC_PLAN_BYTES, KVX_NOALLOC_PARTS_BYTES, arena};
  std::vector<int32_t> pages(50), slots(50);
  for (int i = 0; i < 50; i++) pages[(size_t)i] = slots[(size_t)i] = i;
  std::vector<kvx_work_item> items(4000);
  const float one[2] = {1.0f, 1.0f};
  for (const int32_t dtype : {KVX_KV_BF16, KVX_KV_FP8_E4M3, KVX_KV_FP8_PAGE}) {
    const float* scales = dtype == KVX_KV_FP8_E4M3 ? one : nullptr;
    kvx_pool *p = nullptr, *made = nullptr;
    CHECK(kv_pool_create(64, 16, 2, 64, dtype, scales, scales, &p) == KVX_OK);
    std::vector<std::function<int()>> calls = {
        [&]() { return kv_pool_create(4, 16, 2, 64, dtype, scales, scales, &made); },
        [&]() { return kv_pool_write_pages(p, pages.data(), 50, far_away(1), far_away(2), nullptr); },
        [&]() { return kv_pool_spill(p, pages.data(), slots.data(), 50, far_away(1), 50, nullptr); },
        [&]() { return kv_pool_reload(p, pages.data(), slots.data(), 50, far_away(1), 50, nullptr); },
    };
    for (const TestBatch* t : {&large, &ones, &tiles, &mixed}) {
      calls.push_back([&, t]() { return store_kv(p, &t->b, far_away(1), far_away(2), nullptr); });
      calls.push_back([&, t]() { return store_kv_rope(p, &t->b, &rope, nullptr, 0, nullptr, far_away(1), far_away(2), nullptr); });
      calls.push_back([&, t]() { return load_kv(p, &t->b, far_away(1), far_away(2), nullptr); });
      calls.push_back([&, t]() { return extend_attention(p, &t->b, far_away(1), 6, 0.1f, far_away(2), nullptr, nullptr); });
      calls.push_back([&, t]() { return kvx::attention_call(p, &t->b, far_away(1), 6, 0.1f, far_away(2), nullptr, nullptr, &fixed); });
      calls.push_back([&, t]() { return cross_attention(p, &t->b, far_away(1), 6, 0.1f, far_away(2), nullptr, nullptr); });
      calls.push_back([&, t]() {
        int64_t count = 0;
        return extend_attention_plan(&t->b, 6, 2, 64, 0, items.data(), (int64_t)items.size(), &count);
      });
    }
    for (size_t c = 0; c < calls.size(); c++) {
      int rc = KVX_ENOMEM;
      for (int left = 0; rc == KVX_ENOMEM && left < 10000; left++) {
        g_launches = 0;
        const int blocks = g_device_blocks;
        g_left = left;
        try {
          rc = calls[c]();
        } catch (...) {
          g_left = -1;
          std::fprintf(stderr, "an exception left call %zu, %d allocations in, dtype %d\n", c, left, dtype);
          std::exit(5);
        }
        const bool enough = g_left > 0;
        g_left = -1;
        CHECK(rc == KVX_OK || rc == KVX_ENOMEM);
        if (enough) CHECK(rc == KVX_OK);
        if (rc == KVX_ENOMEM) CHECK(kvx_last_error()[0] != 0 && g_launches == 0);
        if (c == 0) {
          CHECK((rc == KVX_OK) == (made != nullptr));
          if (made) CHECK(kv_pool_destroy(made) == KVX_OK);
          made = nullptr;
          CHECK(g_device_blocks == blocks);  // nothing of a pool that was not made stays
        }
      }
      CHECK(rc == KVX_OK);
    }
    CHECK(kv_pool_destroy(p) == KVX_OK);
  }
  CHECK(g_device_blocks == 0);
}

// What a failed call says is there until the next call, whole up to the longest.
void messages() {
  for (const int n : {0, 3, 15, 16, 300, 511, 512, 5000}) {
    const std::string text((size_t)n, 'x');
    CHECK(kvx::report(KVX_EINVAL, "%s", text.c_str()) == KVX_EINVAL);
    CHECK(std::string(kvx_last_error()) == text.substr(0, 511));
  }
  CHECK(kv_pool_set_split_keys(nullptr, 0) == KVX_EINVAL && std::strcmp(kvx_last_error(), "pool is NULL") == 0);
  kvx_pool* p = nullptr;
  CHECK(kv_pool_create(4, 16, 2, 64, KVX_KV_BF16, nullptr, nullptr, &p) == KVX_OK && kvx_last_error()[0] == 0);
  CHECK(kv_pool_set_split_keys(p, 65) == KVX_EINVAL && kvx_last_error()[0] != 0);
  CHECK(kv_pool_set_split_keys(p, 64) == KVX_OK && kvx_last_error()[0] == 0);
  CHECK(kv_pool_destroy(p) == KVX_OK);
}

// The ranges of a plan of few rows: longest unit and ranges of the longest entry; whether it fits
// the kernel's arguments.
struct Ranges {
  int64_t longest = 0, of_longest = 0;
  bool in_args = false;
};
Ranges ranges_of(const std::vector<RowsRequest>& reqs, int32_t heads, int32_t head_dim, bool bf16) {
  const RowsPlan plan = make_rows_plan(reqs, heads, 1, 2 * head_dim * (bf16 ? 2 : 1), bf16, 0, kMaxParts);
  Ranges r;
  r.in_args = plan.words.size() <= (size_t)kvx::kRowsWords;
  int64_t keys = 0, codes = 0;
  for (size_t i = 0; i < reqs.size(); i++) {
    RowsEntry e;
    std::memcpy(&e, plan.words.data() + i * kvx::kRowsEntryWords, sizeof e);
    CHECK(e.keys == reqs[i].keys && e.len > 0 && e.len % kvx::kDecodeChunkAlign == 0);
    const int64_t n = e.keys > 0 ? (e.keys - 1) / e.len + 1 : 1;
    r.longest = std::max<int64_t>(r.longest, std::min(e.keys, e.len));
    if (e.keys > keys) {
      keys = e.keys;
      r.of_longest = n;
    }
    codes += n;
  }
  CHECK(plan.n_codes == codes && (int64_t)plan.words.size() == codes + (int64_t)reqs.size() * kvx::kRowsEntryWords);
  return r;
}

// Ranges are lengthened for room in the kernel's arguments only where the longest unit's time, at 200 or 120 keys a
// microsecond, grows by less than the copy and the merging that this saves; half of that growth
// may pass where reading all keys takes longer.  With as many entries without keys as leave no room the
// ranges are not lengthened.
void ranges() {
  std::vector<std::vector<int32_t>> lens;
  for (const int n : {1, 60, 100, 130, 132, 133, 134, 135, 200})
    for (const int32_t last : {3000, 30000, 100000, 131072, 262144}) {
      lens.emplace_back((size_t)n, 200);
      lens.back().push_back(last);
    }
  uint32_t rng = 12345;
  auto next = [&]() { return (rng = rng * 1664525u + 1013904223u) >> 8; };
  for (int trial = 0; trial < 400; trial++) {
    lens.emplace_back();
    for (int n = 1 + (int)(next() % 145); n > 0; n--)
      lens.back().push_back((int32_t)std::exp(4.0 + (next() % 1000) / 1000.0 * (trial % 2 ? 6.3 : 4.0)));
  }
  bool fitted = false, copied = false;
  for (const auto& l : lens)
    for (const int32_t heads : {1, 4})
      for (const int32_t head_dim : {64, 128})
        for (const bool bf16 : {false, true}) {
          std::vector<RowsRequest> reqs;
          for (const int32_t keys : l) reqs.push_back(RowsRequest{0, 1, 0, keys});
          const Ranges r = ranges_of(reqs, heads, head_dim, bf16);
          reqs.resize(reqs.size() + 200, RowsRequest{0, 1, 0, 0});
          const Ranges free = ranges_of(reqs, heads, head_dim, bf16);
          const double rate = bf16 ? 120.0 : 200.0, saved = 6.0 + 0.09 * head_dim / 128.0 * (double)free.of_longest;
          CHECK(!free.in_args && r.longest >= free.longest - kvx::kDecodeChunkAlign);
          CHECK((double)(r.longest - free.longest) <= 2.0 * rate * saved + 2 * kvx::kDecodeChunkAlign);
          fitted |= r.longest > free.longest + 64 && r.in_args;
          copied |= !r.in_args && reqs.size() - 200 <= 130;
        }
  CHECK(fitted && copied);  // either choice is made
}

}  // namespace

int main(int argc, char** argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "memory") memory();
  else if (what == "messages") messages();
  else if (what == "ranges") ranges();
  else return 2;
  std::printf("%s passed\n", what.c_str());
  return 0;
}
