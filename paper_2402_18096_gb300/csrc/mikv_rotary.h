// mikv_rotary.h — arguments of the rotary and mask-span kernels (mikv_rotary.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace mikv {

// One tensor of a rotary call: element strides of [batch][heads][tokens][d], input and output.
struct RotaryTensor {
  const void* in;
  void* out;
  long long in_b, in_h, in_t, out_b, out_h, out_t;
  int heads;
};

struct RotaryArgs {
  RotaryTensor x[2];
  const unsigned long long* phases;
  const int32_t* positions;
  int start, batch, tokens, rot;
  int inverse;
  float amplitude;
};

struct SpanArgs {
  int2* spans;
  const int32_t* docs;
  const int32_t* prefix;
  const int32_t* key_len;
  int batch, tq, tk, q_start, causal, n_docs;
};

// vec: 16-byte accesses are possible (alignment of every pointer and stride, whole vectors of turning channels)
cudaError_t launch_rotary(const RotaryArgs& a, int dtype, int layout, bool vec, cudaStream_t st);
cudaError_t launch_mask_spans(const SpanArgs& a, cudaStream_t st);

}  // namespace mikv
