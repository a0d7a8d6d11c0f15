// Attention of trees of new tokens over a paged KV cache: every row sees its request's history, and of the new tokens
// those that its mask names.
#include "attn_ragged_kernels.h"

namespace wam {

hipError_t launch_attn_tree(const RaggedArgs& a, const RaggedPlan& p, void* ws, hipStream_t s) {
  const Parts pt = make_parts(a, p, ws);
  if (a.k_exp) return launch<128, TREE, true>(a, pt, p, s);
  return a.Dh == 128 ? launch<128, TREE, false>(a, pt, p, s) : launch<64, TREE, false>(a, pt, p, s);
}

}  // namespace wam
