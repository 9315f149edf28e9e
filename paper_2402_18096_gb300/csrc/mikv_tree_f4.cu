// mikv_tree_f4.cu — the attention of few drafted rows (mikv_tree_few.cuh) over 4-bit retained codes.
#include "mikv_tree_few.cuh"

namespace mikv {

template <>
cudaError_t launch_tree_few<4>(const TreeFewArgs& p, bool narrow, int grid, cudaStream_t st) {
  return narrow ? tree::launch_few_variant<4, true>(p, grid, st) : tree::launch_few_variant<4, false>(p, grid, st);
}

}  // namespace mikv
