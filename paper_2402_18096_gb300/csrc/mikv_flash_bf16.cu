// mikv_flash_bf16.cu — attention over bf16 keys: instances of the kernel template in mikv_flash.cuh.
#include "mikv_flash.cuh"

namespace mikv {

template <>
cudaError_t launch_flash_kernel<false>(const FlashKernelArgs& p, int mode, int grid, cudaStream_t st) {
  switch (mode) {
    case flash::kPair: return flash::launch_variant<false, flash::kPair>(p, grid, st);
    case flash::kOne: return flash::launch_variant<false, flash::kOne>(p, grid, st);
    case flash::kFew: return flash::launch_variant<false, flash::kFew>(p, grid, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace mikv
