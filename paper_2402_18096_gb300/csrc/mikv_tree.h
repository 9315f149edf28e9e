// mikv_tree.h — arguments of the kernels for drafted tokens (mikv_tree.cu, mikv_path.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mikv_device.cuh"
#include "mikv_internal.h"

namespace mikv {

constexpr int kTreeNodes = MIKV_TREE_NODES;

// [batch][heads][nodes][128] with element strides.
struct TreeView {
  void* p;
  long long b, h, t;
};

// What the requests hold, as mikv_lengths has it, with the limits that the kernels hold it to.
struct HeldArgs {
  const int32_t *n_hi, *n_lo, *slots;
  int hi_cap, n_lo_max;
#ifdef __CUDACC__
  __device__ __forceinline__ int hi(int b) const { return n_hi ? max(0, min(n_hi[b], hi_cap)) : hi_cap; }
  __device__ __forceinline__ int lo(int b) const { return n_lo ? max(0, min(n_lo[b], n_lo_max)) : n_lo_max; }
  // the free slot of KV head bh of request b, or -1
  __device__ __forceinline__ int free_slot(int bh, int hi_used) const {
    if (!slots) return -1;
    const int s = slots[bh];
    return s >= 0 && s < hi_used ? s : -1;
  }
#endif
};

struct TreeArgs {
  TreeView q, k, v, out;
  const __nv_bfloat16 *k_hi, *v_hi;
  const uint8_t *k_codes, *v_codes;
  const __half2 *k_params, *v_params;
  const float* balancer;
  const uint4* masks;  // [batch][nodes]
  float* lse;
  int* status;
  HeldArgs held;
  int batch, heads_q, heads_kv, G, nodes, hi_stride, lo_cap, bits, group;
  float sm_scale;
  int out_f32;
};

// Row numbers, and the costs that the runs are made of, within 32 bits.
bool tree_sizes_ok(const mikv_shape& s, int nodes);
size_t tree_workspace_bytes(const mikv_shape& s, int nodes, int num_sms);
cudaError_t launch_tree_masks(uint4* masks, int32_t* positions, const int32_t* parents, int batch, int nodes,
                              const int32_t* first, int start, cudaStream_t st);
cudaError_t launch_tree(const TreeArgs& a, void* workspace, int num_sms, cudaStream_t st);

struct PathArgs {
  TreeView q, k, v;
  const mikv_cache* cache;
  const int32_t* path;
  const float* lse;
  float* gained;
  const int32_t* first;
  HeldArgs held;
  int32_t *n_hi_out, *n_lo_out, *next;
  int* status;
  int steps, nodes;
  float sm_scale;
};

cudaError_t launch_path_importance(const mikv_shape& s, const PathArgs& a, cudaStream_t st);
cudaError_t launch_commit(const mikv_shape& s, const PathArgs& a, cudaStream_t st);

struct CopyLengths {
  const int32_t *n_hi, *n_lo, *slots;
  int32_t *to_n_hi, *to_n_lo, *to_slots;
  int n_lo_max;
};
cudaError_t launch_copy_requests(const mikv_shape& s, const mikv_cache& c, const mikv_shape& ts, const mikv_cache& tc,
                                 const int32_t* pairs, int n, const CopyLengths& len, cudaStream_t st);

}  // namespace mikv
