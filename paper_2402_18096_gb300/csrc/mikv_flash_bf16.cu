// mikv_flash_bf16.cu — attention over bf16 keys: instances of the kernel template in mikv_flash.cuh.
#include "mikv_flash.cuh"

namespace mikv {

template <>
cudaError_t launch_flash_kernel<false>(const FlashKernelArgs& p, bool pair, int grid, cudaStream_t st) {
  return pair ? flash::launch_variant<false, true>(p, grid, st) : flash::launch_variant<false, false>(p, grid, st);
}

}  // namespace mikv
