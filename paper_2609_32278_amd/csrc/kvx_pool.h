// The KV pool behind the C ABI's opaque handle.
#pragma once

#include "kvx_host_util.h"

struct kvx_pool {
  int device = 0;
  int64_t num_pages = 0;
  int32_t page_size = 16;
  int32_t num_kv_heads = 0;
  int32_t head_dim = 0;
  int32_t kv_dtype = KVX_KV_BF16;
  int32_t elem_bytes = 2;
  void* k = nullptr;
  void* v = nullptr;
  float* scales_d = nullptr;  // [k_scale | v_scale | k_inv | v_inv], each num_kv_heads
  float* page_scales = nullptr;  // page-scaled pool: [num_pages][num_kv_heads][K, V]

  bool page_scaled() const { return kv_dtype == KVX_KV_FP8_PAGE; }
  // The scales that kernels take with the codes: one a head, or every second float one of a
  // page and head.
  float* k_scales() const { return page_scaled() ? page_scales : scales_d; }
  float* v_scales() const {
    if (page_scaled()) return page_scales + 1;
    return scales_d ? scales_d + num_kv_heads : nullptr;
  }
  kvx::Staging st_store, st_load, st_attn, st_io, st_move;
  kvx::Workspace parts;
  int32_t split_keys = 0;  // key-range split length of extend_attention; 0 = automatic
  int32_t scaled_q = 0;    // 1: prefill attention on a bf16 pool takes the folded softmax
};

namespace kvx {

inline int check_pool(const kvx_pool* pool) {
  if (pool == nullptr) return report(KVX_EINVAL, "pool is NULL");
  return KVX_OK;
}

inline int use_device(const kvx_pool* pool) {
  int cur = -1;
  KVX_HIP(hipGetDevice(&cur));
  if (cur != pool->device) KVX_HIP(hipSetDevice(pool->device));
  return KVX_OK;
}

}  // namespace kvx
