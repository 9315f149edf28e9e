// mikv_flash_f16.cu — attention over fp16 keys: instances of the kernel template in mikv_flash.cuh.
#include "mikv_flash.cuh"

namespace mikv {

template <>
cudaError_t launch_flash_kernel<true>(const FlashKernelArgs& p, bool pair, int grid, cudaStream_t st) {
  return pair ? flash::launch_variant<true, true>(p, grid, st) : flash::launch_variant<true, false>(p, grid, st);
}

}  // namespace mikv
