// Prefill attention on a page-scaled pool: the instantiations of the 8-bit kernel in
// kvx_attn_kernels.h that take a power of two a page (PAGE).

#include "kvx_attn_kernels.h"

namespace kvx {

hipError_t launch_page_attention(const AttnParams& p, int64_t n_units, int head_dim, bool scaled_q, hipStream_t stream) {
  if (p.compact != nullptr) launch_attn8<true, false>(p, *p.compact, n_units, head_dim, scaled_q, stream);
  else if (p.mixed) launch_attn8<true, true>(p, UnitsInMemory{}, n_units, head_dim, scaled_q, stream);
  else launch_attn8<true, false>(p, UnitsInMemory{}, n_units, head_dim, scaled_q, stream);
  return hipGetLastError();
}

}  // namespace kvx
