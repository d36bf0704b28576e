// Host code shared by the files behind the C ABI: error returns, upload channels, growable
// device scratch and the checks of a batch.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "kvx.h"
#include "kvx_internal.h"

namespace kvx {

inline int hip_fail(hipError_t e, const char* what) {
  return report(e == hipErrorOutOfMemory ? KVX_ENOMEM : KVX_EHIP, "%s: %s", what, hipGetErrorString(e));
}

#define KVX_HIP(call)                                   \
  do {                                                  \
    hipError_t e_ = (call);                             \
    if (e_ != hipSuccess) return kvx::hip_fail(e_, #call); \
  } while (0)

inline bool validate_mode() {
  const char* v = std::getenv("KVX_VALIDATE");
  return v != nullptr && v[0] != '\0' && v[0] != '0';
}

// Pinned host buffer + device buffer + events: a reusable upload channel.  The
// host side is rewritten only after the previous copy out of it has completed.
// The device buffer grows with the stream-ordered allocator: the old buffer is
// freed in stream order behind `used` (recorded after the last kernels that read
// it), so growing never waits on the host for the device.
struct Staging {
  void* host = nullptr;
  size_t host_cap = 0;
  void* dev = nullptr;
  size_t dev_cap = 0;
  hipEvent_t ev = nullptr;    // after the last copy out of `host`
  hipEvent_t used = nullptr;  // after the last kernels that read `dev`
  bool pending = false;

  // Only after the device has gone idle (pool destruction).
  void release() {
    if (ev) {
      (void)hipEventSynchronize(ev);
      (void)hipEventDestroy(ev);
    }
    if (used) (void)hipEventDestroy(used);
    if (host) (void)hipHostFree(host);
    if (dev) (void)hipFreeAsync(dev, nullptr);
    *this = Staging();
  }

  // Copy `bytes` from `src` to device memory ordered on `stream`; *out receives the
  // device address (valid until the next upload on this channel is ordered after it).
  // The caller records done() on the stream after the kernels that read it.
  int upload(const void* src, size_t bytes, hipStream_t stream, void** out) {
    if (!ev) KVX_HIP(hipEventCreateWithFlags(&ev, hipEventDisableTiming));
    if (!used) KVX_HIP(hipEventCreateWithFlags(&used, hipEventDisableTiming));
    if (pending) {
      KVX_HIP(hipEventSynchronize(ev));
      pending = false;
    }
    if (bytes > host_cap) {
      if (host) KVX_HIP(hipHostFree(host));
      host = nullptr;
      host_cap = 0;
      size_t cap = std::max<size_t>(bytes + bytes / 2, 4096);
      KVX_HIP(hipHostMalloc(&host, cap, hipHostMallocDefault));
      host_cap = cap;
    }
    if (bytes > dev_cap) {
      if (dev) {
        // earlier kernels (on any stream) that read the old buffer precede `used`
        KVX_HIP(hipStreamWaitEvent(stream, used, 0));
        KVX_HIP(hipFreeAsync(dev, stream));
      }
      dev = nullptr;
      dev_cap = 0;
      size_t cap = std::max<size_t>(bytes + bytes / 2, 4096);
      KVX_HIP(hipMallocAsync(&dev, cap, stream));
      dev_cap = cap;
    }
    std::memcpy(host, src, bytes);
    KVX_HIP(hipMemcpyAsync(dev, host, bytes, hipMemcpyHostToDevice, stream));
    KVX_HIP(hipEventRecord(ev, stream));
    pending = true;
    *out = dev;
    return KVX_OK;
  }

  int done(hipStream_t stream) {
    KVX_HIP(hipEventRecord(used, stream));
    return KVX_OK;
  }
};

// Device scratch that only grows, with the same stream-ordered replacement.
struct Workspace {
  void* ptr = nullptr;
  size_t cap = 0;
  hipEvent_t used = nullptr;  // after the last kernels that used `ptr`
  int ensure(size_t bytes, hipStream_t stream) {
    if (!used) KVX_HIP(hipEventCreateWithFlags(&used, hipEventDisableTiming));
    if (bytes <= cap) return KVX_OK;
    if (ptr) {
      KVX_HIP(hipStreamWaitEvent(stream, used, 0));
      KVX_HIP(hipFreeAsync(ptr, stream));
      ptr = nullptr;
      cap = 0;
    }
    // headroom of a quarter for small sizes; past 1 GiB exactly what is asked
    size_t c = bytes > ((size_t)1 << 30) ? bytes : std::max<size_t>(bytes + bytes / 4, 1 << 20);
    KVX_HIP(hipMallocAsync(&ptr, c, stream));
    cap = c;
    return KVX_OK;
  }
  int done(hipStream_t stream) {
    if (used) KVX_HIP(hipEventRecord(used, stream));
    return KVX_OK;
  }
  // Only after the device has gone idle (pool destruction).
  void release() {
    if (ptr) (void)hipFreeAsync(ptr, nullptr);
    if (used) (void)hipEventDestroy(used);
    ptr = nullptr;
    cap = 0;
    used = nullptr;
  }
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The kernels move 16-byte pieces: every bf16 row buffer must start 16-byte aligned.
inline int check_align(const void* ptr, const char* name) {
  if (ptr != nullptr && ((uintptr_t)ptr & 15u) != 0)
    return report(KVX_EINVAL, "%s = %p is not 16-byte aligned", name, ptr);
  return KVX_OK;
}

// Host-side checks of a batch; fills qo offsets (request r owns rows [qo[r], qo[r+1])).
inline int check_batch(const kvx_batch* b, std::vector<int64_t>& qo, bool need_page_ids = true) {
  if (b == nullptr) return report(KVX_EINVAL, "batch is NULL");
  if (b->num_reqs < 0) return report(KVX_EINVAL, "num_reqs = %d < 0", b->num_reqs);
  qo.assign((size_t)b->num_reqs + 1, 0);
  if (b->num_reqs == 0) return KVX_OK;
  if (!b->prefix_lens || !b->extend_lens || !b->page_indptr)
    return report(KVX_EINVAL, "prefix_lens, extend_lens and page_indptr must be non-NULL");
  if (b->page_indptr[0] != 0) return report(KVX_EINVAL, "page_indptr[0] = %d, must be 0", b->page_indptr[0]);
  for (int r = 0; r < b->num_reqs; r++) {
    const int64_t P = b->prefix_lens[r], E = b->extend_lens[r];
    if (P < 0 || E < 0) return report(KVX_EINVAL, "request %d: negative length (P=%lld, E=%lld)", r, (long long)P, (long long)E);
    if (P + E > (int64_t)INT32_MAX - 1024) return report(KVX_EINVAL, "request %d: sequence too long", r);
    const int64_t have = (int64_t)b->page_indptr[r + 1] - b->page_indptr[r];
    if (have < ceil_div(P + E, kPageSize))
      return report(KVX_EINVAL, "request %d: %lld page ids for %lld tokens (need %lld)", r, (long long)have,
                  (long long)(P + E), (long long)ceil_div(P + E, kPageSize));
    qo[r + 1] = qo[r] + E;
  }
  if (qo.back() > (int64_t)INT32_MAX) return report(KVX_EINVAL, "total extend length exceeds 2^31-1");
  if (need_page_ids && b->page_indptr[b->num_reqs] > 0 && b->page_ids == nullptr)
    return report(KVX_EINVAL, "page_ids is NULL");
  return KVX_OK;
}

// KVX_VALIDATE=1: copy the page table to the host and check every id.
inline int check_page_ids(int64_t num_pages, const kvx_batch* b, hipStream_t stream) {
  const int64_t n = b->num_reqs ? b->page_indptr[b->num_reqs] : 0;
  if (n == 0) return KVX_OK;
  std::vector<int32_t> ids((size_t)n);
  KVX_HIP(hipStreamSynchronize(stream));
  KVX_HIP(hipMemcpy(ids.data(), b->page_ids, (size_t)n * sizeof(int32_t), hipMemcpyDeviceToHost));
  for (int64_t i = 0; i < n; i++)
    if (ids[(size_t)i] < 0 || ids[(size_t)i] >= num_pages)
      return report(KVX_ERANGE, "page_ids[%lld] = %d outside [0, %lld)", (long long)i, ids[(size_t)i],
                  (long long)num_pages);
  return KVX_OK;
}

// The requests of a store batch in the kernel arguments when there are few enough
// (returns false otherwise: the unit list is uploaded instead).  Workgroup order
// matches the unit lists below: request by request, logical page by page.
inline bool inline_store_reqs(const kvx_batch* b, const std::vector<int64_t>& qo, StoreReqs& rq) {
  rq.n = 0;
  int32_t wg = 0;
  for (int r = 0; r < b->num_reqs; r++) {
    const int64_t P = b->prefix_lens[r], E = b->extend_lens[r];
    if (E == 0) continue;
    if (rq.n == kStoreInlineReqs) {
      rq.n = 0;
      return false;
    }
    const int64_t pages = (P + E - 1) / kPageSize - P / kPageSize + 1;
    rq.first[rq.n] = wg;
    rq.qo[rq.n] = (int32_t)qo[(size_t)r];
    rq.prefix[rq.n] = (int32_t)P;
    rq.end[rq.n] = (int32_t)(P + E);
    rq.page_base[rq.n] = b->page_indptr[r];
    wg += (int32_t)pages;
    rq.n++;
  }
  rq.first[rq.n] = wg;
  return rq.n > 0;
}

}  // namespace kvx
