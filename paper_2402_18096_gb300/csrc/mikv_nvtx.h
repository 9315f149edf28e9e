// mikv_nvtx.h — one NVTX range per compute entry point of the C ABI.
#pragma once

#ifndef MIKV_NVTX
#define MIKV_NVTX 1
#endif
#if MIKV_NVTX
#include <nvtx3/nvToolsExt.h>
#endif

namespace mikv {

// One NVTX range per compute entry point, named after the call, around its validation and launches (host time:
// the kernels run later on the stream). Without a tool attached, push and pop return at once; -DMIKV_NVTX=0
// leaves them out.
struct CallRange {
#if MIKV_NVTX
  explicit CallRange(const char* name) { nvtxRangePushA(name); }
  ~CallRange() { nvtxRangePop(); }
#else
  explicit CallRange(const char*) {}
#endif
  CallRange(const CallRange&) = delete;
  CallRange& operator=(const CallRange&) = delete;
};

}  // namespace mikv

#define MIKV_CALL_RANGE() const ::mikv::CallRange mikv_call_range_(__func__)
