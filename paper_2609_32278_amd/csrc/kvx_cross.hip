// Cross attention through tiles: the instantiations of the prefill kernels in
// kvx_attn_kernels.h whose rows all see every key of their unit.  A tile's rows stand at the
// request's last key, so that the causal mask leaves out what lies past it and nothing else.
// 8 requests of 30 to 1200 queries on 1030 to 6200 tokens, page-scaled pool, 32/8/128 heads: 125 us a call,
// where the products of the queries take 80 at 1220 TFLOP/s and the busiest CU's 60 steps of 64 keys (50 in
// the mean, 92% of the rows queries) 106; each unit waits for its first tiles.

#include "kvx_attn_kernels.h"

namespace kvx {

hipError_t launch_cross_attention(const AttnParams& p, int64_t n_units, int head_dim, bool fp8, bool scaled_q,
                                  hipStream_t stream) {
  auto launch = [&](const auto& plan) {
    if (fp8) launch_attn8<false, false>(p, plan, n_units, head_dim, scaled_q, stream);
    else launch_attn<false>(p, plan, n_units, head_dim, false, scaled_q, stream);
  };
  if (p.compact != nullptr) launch(CrossCompactPlan{*p.compact});
  else launch(CrossUnitsInMemory{});
  return hipGetLastError();
}

}  // namespace kvx
