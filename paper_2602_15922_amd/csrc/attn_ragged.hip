// Attention of ragged rows over a paged KV cache, or over packed states of other lengths.
#include "attn_ragged_kernels.h"

namespace wam {

hipError_t launch_attn_ragged(const RaggedArgs& a, const RaggedPlan& p, void* ws, hipStream_t s) {
  const Parts pt = make_parts(a, p, ws);
  if (a.table) {
    if (a.k_exp) return launch<128, PAGES, true>(a, pt, p, s);
    return a.Dh == 128 ? launch<128, PAGES, false>(a, pt, p, s) : launch<64, PAGES, false>(a, pt, p, s);
  }
  return a.Dh == 128 ? launch<128, STATES, false>(a, pt, p, s) : launch<64, STATES, false>(a, pt, p, s);
}

}  // namespace wam
