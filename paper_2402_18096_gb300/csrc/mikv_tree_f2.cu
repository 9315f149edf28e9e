// mikv_tree_f2.cu — the attention of few drafted rows (mikv_tree_few.cuh) over 2-bit retained codes, and over caches without a
// retained set.
#include "mikv_tree_few.cuh"

namespace mikv {

template <>
cudaError_t launch_tree_few<2>(const TreeFewArgs& p, bool narrow, int grid, cudaStream_t st) {
  return narrow ? tree::launch_few_variant<2, true>(p, grid, st) : tree::launch_few_variant<2, false>(p, grid, st);
}

}  // namespace mikv
