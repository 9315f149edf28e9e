// mikv_tree.cu — drafted tokens: what the nodes of a tree see of one another, and their attention over the
// mixed-precision cache.
#include <math.h>

#include "mikv_quant_rows.cuh"
#include "mikv_tree.h"

namespace mikv {
namespace {

// One block per request: every thread walks from its node up to the root through the parents in shared memory (128 steps
// at most; a chain of 128 takes 4 us, and the masks serve all layers of a step).
__global__ void __launch_bounds__(kTreeNodes) tree_masks_kernel(uint4* masks, int32_t* positions, const int32_t* parents,
                                                                int nodes, const int32_t* first, int start) {
  __shared__ int up[kTreeNodes];
  const int b = blockIdx.x, i = threadIdx.x;
  grid_dependency_wait();
  allow_dependent_launch();
  if (i < nodes) up[i] = parents[(size_t)b * nodes + i];
  __syncthreads();
  if (i >= nodes) return;
  uint32_t m[4] = {0u, 0u, 0u, 0u};
  int depth = -1;
  for (int j = i; j >= 0;) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if ((j >> 5) == w) m[w] |= 1u << (j & 31);
    ++depth;
    const int p = up[j];
    if (p < -1 || p >= j) {  // no node, or below one that is none
      depth = -1;
      break;
    }
    j = p;
  }
  const bool node = depth >= 0;
  masks[(size_t)b * nodes + i] = node ? make_uint4(m[0], m[1], m[2], m[3]) : make_uint4(0u, 0u, 0u, 0u);
  if (positions) positions[(size_t)b * nodes + i] = (first ? first[b] : start) + max(depth, 0);
}

// The code of channel c in a packed row.
__device__ __forceinline__ int code_at(const uint8_t* row, int bits, int c) {
  const uint16_t* units = reinterpret_cast<const uint16_t*>(row);
  int unit, bit;
  field_pos(c, bits == 3 ? 2 : bits, unit, bit);
  int code = (units[unit] >> bit) & (bits == 4 ? 15 : 3);
  if (bits == 3) {
    field_pos(c, 1, unit, bit);
    code |= ((units[16 + unit] >> bit) & 1) << 2;
  }
  return code;
}

__device__ __forceinline__ void bf16x4(const __nv_bfloat16* p, float (&x)[4]) {
  const uint2 r = *reinterpret_cast<const uint2*>(p);
  x[0] = __uint_as_float(r.x << 16);
  x[1] = __uint_as_float(r.x & 0xffff0000u);
  x[2] = __uint_as_float(r.y << 16);
  x[3] = __uint_as_float(r.y & 0xffff0000u);
}

// One block per (node, query head, request), a key to a warp at a time, all in fp32.
__global__ void __launch_bounds__(128) tree_rows_kernel(const TreeArgs a) {
  __shared__ float s_o[4][kHeadDim], s_m[4], s_l[4];
  __shared__ int s_bad;
  const int node = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = hq / a.G, bh = b * a.heads_kv + h;
  const uint4 mw = a.masks[(size_t)b * a.nodes + node];
  const uint32_t mask[4] = {mw.x, mw.y, mw.z, mw.w};
  const bool real = mask[node >> 5] >> (node & 31) & 1;
  const int n_hi = a.held.hi(b), n_lo = a.held.lo(b), free_slot = a.held.free_slot(bh, n_hi);
  float q[4], qb[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  bf16x4(static_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + hq * a.q.h + node * a.q.t + 4 * lane, q);
#pragma unroll
  for (int e = 0; e < 4; ++e) qb[e] = a.balancer ? q[e] / a.balancer[h * kHeadDim + 4 * lane + e] : q[e];
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  for (int t = warp; real && t < n_hi + n_lo + a.nodes; t += 4) {
    float k[4], v[4];
    const float* x = q;
    if (t < n_hi) {
      if (t == free_slot) continue;
      const size_t row = ((size_t)bh * a.hi_stride + t) * kHeadDim + 4 * lane;
      bf16x4(a.k_hi + row, k);
      bf16x4(a.v_hi + row, v);
    } else if (t < n_hi + n_lo) {
      const size_t row = (size_t)bh * a.lo_cap + (t - n_hi);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 4 * lane + e;
        const float2 kp = __half22float2(a.k_params[row * (kHeadDim / a.group) + c / a.group]);
        const float2 vp = __half22float2(a.v_params[row * (kHeadDim / a.group) + c / a.group]);
        k[e] = fmaf(kp.x, (float)code_at(a.k_codes + row * 16 * a.bits, a.bits, c), kp.y);
        v[e] = fmaf(vp.x, (float)code_at(a.v_codes + row * 16 * a.bits, a.bits, c), vp.y);
      }
      x = qb;
    } else {
      const int j = t - n_hi - n_lo;
      if (!(mask[j >> 5] >> (j & 31) & 1)) continue;
      bf16x4(static_cast<const __nv_bfloat16*>(a.k.p) + b * a.k.b + h * a.k.h + j * a.k.t + 4 * lane, k);
      bf16x4(static_cast<const __nv_bfloat16*>(a.v.p) + b * a.v.b + h * a.v.h + j * a.v.t + 4 * lane, v);
      if (!(isfinite(v[0]) && isfinite(v[1]) && isfinite(v[2]) && isfinite(v[3]))) s_bad = 1;
    }
    float s = x[0] * k[0] + x[1] * k[1] + x[2] * k[2] + x[3] * k[3];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    s *= a.sm_scale;
    const float top = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - top), w = s == -INFINITY ? 0.f : expf(s - top);
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = o[e] * f + w * v[e];
    m = top;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) s_o[warp][4 * lane + e] = o[e];
  if (lane == 0) s_m[warp] = m, s_l[warp] = l;
  __syncthreads();
  const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  float total = 0.f, y = 0.f;
  const int c = threadIdx.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f = s_m[i] == -INFINITY ? 0.f : expf(s_m[i] - top);
    total += s_l[i] * f;
    y += f == 0.f ? 0.f : s_o[i][c] * f;
  }
  y = !real ? 0.f : s_bad ? __int_as_float(0x7fffffff) : y / total;
  const long long at = b * a.out.b + hq * a.out.h + node * a.out.t + c;
  if (a.out_f32)
    static_cast<float*>(a.out.p)[at] = y;
  else
    static_cast<__nv_bfloat16*>(a.out.p)[at] = __float2bfloat16(y);
  if (a.lse && c == 0)
    a.lse[((size_t)b * a.heads_q + hq) * a.nodes + node] = real ? top + logf(total) : -INFINITY;
}

}  // namespace

cudaError_t launch_tree_masks(uint4* masks, int32_t* positions, const int32_t* parents, int batch, int nodes,
                              const int32_t* first, int start, cudaStream_t st) {
  return launch_chained(tree_masks_kernel, dim3(batch), dim3(kTreeNodes), 0, st, masks, positions, parents, nodes, first,
                        start);
}

size_t tree_workspace_bytes(const mikv_shape&, int, int) { return kWsHeader; }

cudaError_t launch_tree(const TreeArgs& a, void*, int, cudaStream_t st) {
  tree_rows_kernel<<<dim3(a.nodes, a.heads_q, a.batch), 128, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace mikv
