// mikv_tree_f3.cu — the attention of few drafted rows (mikv_tree_few.cuh) over 3-bit retained codes.
#include "mikv_tree_few.cuh"

namespace mikv {

template <>
cudaError_t launch_tree_few<3>(const TreeFewArgs& p, bool narrow, int grid, cudaStream_t st) {
  return narrow ? tree::launch_few_variant<3, true>(p, grid, st) : tree::launch_few_variant<3, false>(p, grid, st);
}

}  // namespace mikv
