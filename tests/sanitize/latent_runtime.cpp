// Checks of latent attention's host code (csrc/kvx_latent_host.cpp) over a stand-in for the HIP
// runtime with two devices, whose allocations can be made to fail: what a call does with streams,
// devices and errors.  Built by tests/test_latent_runtime.py with the sanitizers; kernels are not
// launched but counted.  The argument names the check.

#include "kvx_latent_host.cpp"

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <set>
#include <string>

struct ihipStream_t {
  int device;
};

namespace fake {
int current = 0;
int fail_host = 0, fail_device = 0;  // how many of the next allocations fail
hipError_t last = hipSuccess;
std::vector<std::string> launched;
std::vector<int> launched_on;
std::set<void*> host;  // live pinned buffers

hipError_t done(hipError_t e) {
  if (e != hipSuccess) last = e;
  return e;
}
}  // namespace fake

extern "C" {
hipError_t hipGetDevice(int* d) { return *d = fake::current, hipSuccess; }
hipError_t hipSetDevice(int d) { return fake::current = d, hipSuccess; }
hipError_t hipGetLastError() {
  const hipError_t e = fake::last;
  fake::last = hipSuccess;
  return e;
}
const char* hipGetErrorString(hipError_t) { return "stand-in error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* st) {
  return *st = hipStreamCaptureStatusNone, hipSuccess;
}
hipError_t hipStreamGetDevice(hipStream_t s, hipDevice_t* d) { return *d = s->device, hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return *e = (hipEvent_t)std::malloc(1), hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t e) { return std::free((void*)e), hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipHostMalloc(void** p, size_t n, unsigned) {
  if (fake::fail_host > 0) return fake::fail_host--, fake::done(hipErrorOutOfMemory);
  *p = std::malloc(n);
  fake::host.insert(*p);
  return hipSuccess;
}
hipError_t hipHostFree(void* p) { return fake::host.erase(p), std::free(p), hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { return *p = std::malloc(n), hipSuccess; }
hipError_t hipFree(void* p) { return std::free(p), hipSuccess; }
hipError_t hipMallocAsync(void** p, size_t n, hipStream_t) {
  if (fake::fail_device > 0) return fake::fail_device--, fake::done(hipErrorOutOfMemory);
  // workspaces are never touched here: their size is not reserved
  return *p = std::malloc(n < (1 << 20) ? n : 64), hipSuccess;
}
hipError_t hipFreeAsync(void* p, hipStream_t) { return std::free(p), hipSuccess; }
hipError_t hipMemset(void* p, int v, size_t n) { return std::memset(p, v, n), hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { return std::memcpy(d, s, n), hipSuccess; }
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) {
  return std::memcpy(d, s, n), hipSuccess;
}
}

namespace kvx {
static std::string g_message;
int report(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_message = buf;
  return code;
}
static hipError_t count(const char* name) {
  fake::launched.push_back(name);
  fake::launched_on.push_back(fake::current);
  return hipSuccess;
}
hipError_t launch_store_latent(const LatentStoreParams&, int64_t, int, bool, bool, hipStream_t) { return count("store"); }
hipError_t launch_load_latent(const LatentLoadParams&, int64_t, int, bool, hipStream_t) { return count("load"); }
hipError_t launch_latent_attention(const LatentAttnParams&, int64_t, const LatentSmallPlan*, const LatentRowPlan*, int,
                                   bool, int, hipStream_t) {
  return count("attention");
}
hipError_t launch_latent_merge(const LatentMergeParams&, int64_t, const LatentSmallPlan*, const LatentRowPlan*, int, int,
                               hipStream_t) {
  return count("merge");
}
hipError_t launch_latent_absorb(const LatentProjParams&, int64_t, int, int, hipStream_t) { return count("absorb"); }
hipError_t launch_latent_output(const LatentProjParams&, int64_t, int, int, hipStream_t) { return count("output"); }
hipError_t launch_latent_expand(const LatentExpandParams&, int64_t, int, int, bool, hipStream_t) { return count("expand"); }
hipError_t launch_latent_prefill(const LatentPrefillParams&, int64_t, int, hipStream_t) { return count("prefill"); }
hipError_t launch_latent_tile_merge(const LatentTileMergeParams&, int64_t, int, hipStream_t) { return count("tiles"); }
}  // namespace kvx

#define CHECK(cond)                                                                                        \
  do {                                                                                                     \
    if (!(cond)) {                                                                                         \
      std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #cond, kvx::g_message.c_str()); \
      std::exit(3);                                                                                        \
    }                                                                                                      \
  } while (0)

namespace {

struct TestBatch {
  std::vector<int32_t> P, E, indptr{0};
  int32_t ids = 0;
  kvx_batch b{};
  void add(int32_t p, int32_t e) {
    P.push_back(p);
    E.push_back(e);
    indptr.push_back(indptr.back() + (int32_t)(((int64_t)p + e + 15) / 16));
  }
  const kvx_batch* get() {
    b = kvx_batch{(int32_t)P.size(), P.data(), E.data(), indptr.data(), &ids};
    return &b;
  }
};

void* addr(uintptr_t a) { return (void*)a; }

kvx_latent_pool* make_pool(int device) {
  const int before = fake::current;
  fake::current = device;
  kvx_latent_pool* p = nullptr;
  CHECK(latent_pool_create(4, 16, 256, 64, KVX_LATENT_BF16, &p) == KVX_OK);
  fake::current = before;
  return p;
}

// Every call on a pool of device 1, with device 0 current.
std::vector<int> all_calls(kvx_latent_pool* pool, const kvx_batch* b, hipStream_t s) {
  const kvx_rope rope{10000.0, nullptr, 64, KVX_ROPE_HALF, nullptr, nullptr, 1e-6f};
  const kvx_latent_proj proj{addr(0x300000), addr(0x400000), 4, 64, 64};
  void *x = addr(0x10000), *q = addr(0x100000), *o = addr(0x200000);
  return {store_latent(pool, b, x, 320, s),
          store_latent_rope(pool, b, &rope, nullptr, 0, 0, nullptr, x, 320, s),
          load_latent(pool, b, x, 320, s),
          latent_attention(pool, b, q, 4, 0.1f, o, nullptr, s),
          latent_extend_attention(pool, b, &proj, q, 0.1f, o, nullptr, KVX_LATENT_ABSORBED, s),
          latent_extend_attention(pool, b, &proj, q, 0.1f, o, nullptr, KVX_LATENT_EXPANDED, s)};
}

// A stream of another device than the pool's is refused; the pool's own and the null stream run
// there, and the caller's device stays current.
void streams() {
  kvx_latent_pool* pool = make_pool(1);
  TestBatch t;
  t.add(20, 3);
  ihipStream_t other{0}, own{1};
  for (int rc : all_calls(pool, t.get(), &other)) CHECK(rc == KVX_EINVAL);
  CHECK(fake::launched.empty() && fake::current == 0);
  for (hipStream_t s : {&own, (ihipStream_t*)nullptr})
    for (int rc : all_calls(pool, t.get(), s)) CHECK(rc == KVX_OK);
  CHECK(!fake::launched.empty() && fake::current == 0);
  for (int d : fake::launched_on) CHECK(d == 1);
  CHECK(latent_pool_destroy(pool) == KVX_OK && fake::current == 0);
}

// After an upload whose buffers could not be had, on the host or on the device, the pool works on.
void staging() {
  kvx_latent_pool* pool = make_pool(0);
  TestBatch some, more;
  for (int i = 0; i < kvx::kStoreInlineReqs + 1; i++) some.add(i, 1);
  for (int i = 0; i < 4000; i++) more.add(i, 1);
  void* x = addr(0x10000);
  CHECK(store_latent(pool, some.get(), x, 320, nullptr) == KVX_OK);
  for (int* failing : {&fake::fail_host, &fake::fail_device}) {
    *failing = 1;
    fake::launched.clear();
    CHECK(store_latent(pool, more.get(), x, 320, nullptr) == KVX_ENOMEM && fake::launched.empty());
    CHECK(*failing == 0 && fake::last == hipSuccess);
    CHECK(store_latent(pool, some.get(), x, 320, nullptr) == KVX_OK && fake::launched.size() == 1);
  }
  CHECK(store_latent(pool, more.get(), x, 320, nullptr) == KVX_OK);
  CHECK(latent_pool_destroy(pool) == KVX_OK && fake::host.empty());
}

// Tokens whose expansion one call cannot index: the expanded form is refused, the automatic
// choice takes the other.
void many_tokens() {
  kvx_latent_pool* pool = make_pool(0);
  TestBatch t;
  for (int i = 0; i < 2; i++) t.add(1100000000, 600);
  const kvx_latent_proj proj{addr(0x300000), addr(0x400000), 4, 64, 64};
  auto call = [&](int form) {
    fake::launched.clear();
    return latent_extend_attention(pool, t.get(), &proj, addr(0x100000), 0.1f, addr(0x800000), nullptr, form, nullptr);
  };
  CHECK(call(KVX_LATENT_EXPANDED) == KVX_EUNSUPPORTED && fake::launched.empty());
  CHECK(call(KVX_LATENT_AUTO) == KVX_OK);
  CHECK(fake::launched == (std::vector<std::string>{"absorb", "attention", "merge", "output"}));
  CHECK(latent_pool_destroy(pool) == KVX_OK);
}

// The automatic choice takes the form that was measured to be faster by a fifth or more (us,
// absorbed and expanded): whole tiles, units and pool types count.
void choices() {
  struct Timed {
    int lat, hd, heads;
    bool fp8;
    int reqs, prefix, extend;
    double absorbed, expanded;
  };
  const Timed timed[] = {
      {512, 128, 16, false, 12, 8000, 128, 470.8, 673.7},  {512, 128, 16, false, 12, 8000, 512, 1545.3, 979.6},
      {512, 128, 16, true, 12, 8000, 180, 821.1, 662.3},   {512, 128, 16, true, 12, 8000, 300, 1158.7, 911.2},
      {256, 128, 64, false, 4, 3000, 400, 507.3, 412.1},   {256, 128, 64, true, 4, 3000, 400, 601.5, 409.2},
      {256, 128, 16, false, 12, 8000, 257, 617.8, 772.0},  {256, 128, 16, true, 2, 30000, 400, 687.3, 446.8},
      {256, 64, 16, false, 12, 8000, 300, 614.7, 484.2},   {512, 64, 16, false, 12, 8000, 257, 938.2, 578.5},
      {512, 128, 4, false, 6, 500, 1, 28.8, 45.5},         {256, 128, 4, true, 6, 500, 1, 25.4, 37.3},
      {512, 128, 96, true, 9, 562, 136, 473.0, 317.0},     {256, 128, 37, true, 22, 126, 2, 28.0, 71.0},
  };
  for (const Timed& t : timed) {
    TestBatch b;
    for (int i = 0; i < t.reqs; i++) b.add(t.prefix, t.extend);
    for (bool absorbed : choose_forms(b.get(), t.heads, t.lat, t.hd, t.fp8))
      if (absorbed != (t.absorbed < t.expanded)) {
        std::fprintf(stderr, "latent %d, %d heads of %d, %d + %d tokens\n", t.lat, t.heads, t.hd, t.prefix, t.extend);
        std::exit(3);
      }
  }
}

// Outputs that overlap an input, which other workgroups may still read, or each other.
void overlaps() {
  kvx_latent_pool* pool = make_pool(0);
  TestBatch t;
  t.add(20, 3);
  const kvx_batch* b = t.get();
  const kvx_rope rope{10000.0, nullptr, 64, KVX_ROPE_HALF, nullptr, nullptr, 1e-6f};
  const uintptr_t q = 0x100000, kv = 0x300000;
  const uintptr_t q_bytes = 3 * 4 * 128 * 2;
  auto store = [&](uintptr_t q_out, int64_t stride) {
    return store_latent_rope(pool, b, &rope, addr(q), 4, 128, addr(q_out), addr(kv), stride, nullptr);
  };
  CHECK(store(kv, 320) == KVX_EINVAL);
  CHECK(store(kv - q_bytes + 16, 320) == KVX_EINVAL && store(kv - q_bytes, 320) == KVX_OK);
  CHECK(store(kv + 3 * 640 - 16, 320) == KVX_EINVAL && store(kv + 3 * 640, 320) == KVX_OK);
  CHECK(store(kv + 640, 4096) == KVX_OK);            // between two rows: 3072 bytes of 7552
  CHECK(store(kv + 8192 - q_bytes, 4096) == KVX_OK);
  CHECK(store(kv + 624, 4096) == KVX_EINVAL && store(kv + 8192 - q_bytes + 16, 4096) == KVX_EINVAL);
  CHECK(store(kv + 2 * 8192 + 640, 4096) == KVX_OK && store(kv + 2 * 8192 + 624, 4096) == KVX_EINVAL);
  auto attend = [&](uintptr_t out, uintptr_t lse) {
    return latent_attention(pool, b, addr(q), 4, 0.1f, addr(out), (float*)lse, nullptr);
  };
  const uintptr_t rows = 3 * 4, o = 0x200000;
  CHECK(attend(q, 0) == KVX_EINVAL && attend(q + rows * 640 - 16, 0) == KVX_EINVAL);
  CHECK(attend(q - rows * 512 + 16, 0) == KVX_EINVAL && attend(q - rows * 512, 0) == KVX_OK);
  CHECK(attend(q + rows * 640, 0) == KVX_OK);
  CHECK(attend(o, q + 64) == KVX_EINVAL && attend(o, o) == KVX_EINVAL && attend(o, o + rows * 512 - 4) == KVX_EINVAL);
  CHECK(attend(o, o + rows * 512) == KVX_OK && attend(o, o - rows * 4) == KVX_OK);
  const uintptr_t uk = 0x400000, uv = 0x500000, w_bytes = 4 * 64 * 256 * 2;
  const kvx_latent_proj proj{addr(uk), addr(uv), 4, 64, 64};
  auto extend = [&](uintptr_t out, uintptr_t lse) {
    return latent_extend_attention(pool, b, &proj, addr(q), 0.1f, addr(out), (float*)lse, KVX_LATENT_AUTO, nullptr);
  };
  CHECK(extend(q + 16, 0) == KVX_EINVAL && extend(uk + w_bytes - 16, 0) == KVX_EINVAL && extend(uv, 0) == KVX_EINVAL);
  CHECK(extend(o, uk) == KVX_EINVAL && extend(o, uv + 16) == KVX_EINVAL && extend(o, o + 16) == KVX_EINVAL);
  CHECK(extend(o, q) == KVX_EINVAL && extend(o, o + rows * 128) == KVX_OK && extend(q + rows * 256, uv + w_bytes) == KVX_OK);
  CHECK(latent_pool_destroy(pool) == KVX_OK);
}

}  // namespace

int main(int argc, char** argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "streams") streams();
  else if (what == "staging") staging();
  else if (what == "tokens") many_tokens();
  else if (what == "choices") choices();
  else if (what == "overlaps") overlaps();
  else return 2;
  std::printf("%s passed\n", what.c_str());
  return 0;
}
