// load_kv: tokens of a KV pool read back as rows (include/kvx.h).

#include "kvx_pool.h"

using kvx::check_align;
using kvx::meet;
using kvx::report;

extern "C" int load_kv(const kvx_pool* pool, const kvx_batch* batch, void* k_out, void* v_out, kvx_stream_t stream) {
  return kvx::guarded([&]() -> int {
    if (int rc = kvx::check_pool(pool)) return rc;
    std::vector<int64_t> qo;
    if (int rc = kvx::check_batch(batch, qo)) return rc;
    if (int rc = check_align(k_out, "k_out")) return rc;
    if (int rc = check_align(v_out, "v_out")) return rc;
    if (qo.back() == 0) return KVX_OK;
    if (!k_out || !v_out) return report(KVX_EINVAL, "k_out and v_out must be non-NULL");
    const size_t bytes = (size_t)qo.back() * pool->num_kv_heads * pool->head_dim * 2;
    if (meet(k_out, bytes, v_out, bytes)) return report(KVX_EINVAL, "k_out overlaps v_out");
    hipStream_t s = (hipStream_t)stream;
    kvx::OnDevice on;
    if (int rc = on.enter(pool->device)) return rc;
    if (int rc = kvx::check_stream(s, pool->device)) return rc;
    if (kvx::validate_mode())
      if (int rc = kvx::check_page_ids(pool->num_pages, batch, s)) return rc;
    kvx::LoadParams p{};
    kvx::Staging& units = const_cast<kvx_pool*>(pool)->st_load;
    int64_t n_units = 0;
    if (int rc = kvx::check_grid(kvx::touched_pages(batch))) return rc;
    if (int rc = kvx::place_units(units, batch, qo, s, p, n_units)) return rc;
    p.k_pool = pool->k;
    p.v_pool = pool->v;
    p.k_scale = pool->k_scales();
    p.v_scale = pool->v_scales();
    p.page_scale = pool->page_scales;
    p.k_out = (uint16_t*)k_out;
    p.v_out = (uint16_t*)v_out;
    p.page_ids = batch->page_ids;
    p.num_kv_heads = pool->num_kv_heads;
    const hipError_t e = kvx::launch_load_kv(p, n_units, pool->head_dim, pool->kv_dtype, s);
    if (e != hipSuccess) return kvx::hip_fail(e, "load_kv kernel launch");
    return KVX_OK;
  });
}
