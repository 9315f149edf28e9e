// mikv_tree_b4.cu — the attention of drafted tokens (mikv_tree_kernel.cuh) over 4-bit retained codes.
#include "mikv_tree_kernel.cuh"

namespace mikv {

template <>
cudaError_t launch_tree_kernel<4>(const TreeKernelArgs& p, bool pair, int grid, cudaStream_t st) {
  return pair ? tree::launch_variant<4, true>(p, grid, st) : tree::launch_variant<4, false>(p, grid, st);
}

}  // namespace mikv
