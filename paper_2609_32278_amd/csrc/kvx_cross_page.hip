// Cross attention through tiles on a page-scaled pool (see kvx_cross.hip).

#include "kvx_attn_kernels.h"

namespace kvx {

hipError_t launch_cross_page_attention(const AttnParams& p, int64_t n_units, int head_dim, bool scaled_q,
                                       hipStream_t stream) {
  if (p.compact != nullptr)
    launch_attn8<true, false>(p, CrossCompactPlan{*p.compact}, n_units, head_dim, scaled_q, stream);
  else
    launch_attn8<true, false>(p, CrossUnitsInMemory{}, n_units, head_dim, scaled_q, stream);
  return hipGetLastError();
}

}  // namespace kvx
