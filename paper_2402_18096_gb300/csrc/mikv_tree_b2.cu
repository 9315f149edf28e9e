// mikv_tree_b2.cu — the attention of drafted tokens (mikv_tree_kernel.cuh) over 2-bit retained codes, and over caches
// without a retained set.
#include "mikv_tree_kernel.cuh"

namespace mikv {

template <>
cudaError_t launch_tree_kernel<2>(const TreeKernelArgs& p, bool pair, int grid, cudaStream_t st) {
  return pair ? tree::launch_variant<2, true>(p, grid, st) : tree::launch_variant<2, false>(p, grid, st);
}

}  // namespace mikv
