// The tree attention's kernels for bf16 queries.
#include "tree_wide.h"

namespace emoe {

void launch_tree_bf16(const TreeArg& a, const TreePlan& p, int head_dim, bool e4m3, hipStream_t stream) {
  if (e4m3) launch_tree<Bf16, true>(a, p, head_dim, stream);
  else launch_tree<Bf16, false>(a, p, head_dim, stream);
}

}  // namespace emoe
