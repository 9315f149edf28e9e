// mikv_flash_f16.cu — attention over fp16 keys: instances of the kernel template in mikv_flash.cuh.
#include "mikv_flash.cuh"

namespace mikv {

template <>
cudaError_t launch_flash_kernel<true>(const FlashKernelArgs& p, int mode, int grid, cudaStream_t st) {
  switch (mode) {
    case flash::kPair: return flash::launch_variant<true, flash::kPair>(p, grid, st);
    case flash::kOne: return flash::launch_variant<true, flash::kOne>(p, grid, st);
    case flash::kFew: return flash::launch_variant<true, flash::kFew>(p, grid, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace mikv
