// mikv_flash.cu — attention over bf16 / fp16 keys (sm_103a): prompts, and single tokens over a shared prefix.
//
// One block per (set of keys, query head, token): 128 keys at a time, a thread per key for the scores and a thread
// per channel for the output, online softmax in fp32. Masked keys are never read.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "mikv_flash.h"

namespace mikv {
namespace {

constexpr float kLn2 = 0.6931471805599453f;

template <bool F16>
__device__ __forceinline__ float load16(const void* p, long long i) {
  return F16 ? __half2float(static_cast<const __half*>(p)[i]) : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

template <bool F16, bool OUT32>
__global__ void __launch_bounds__(128) flash_rows_kernel(const __grid_constant__ FlashArgs a) {
  __shared__ float s_q[128], s_p[128], s_red[4];
  const int tid = threadIdx.x, t = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int kv = h / a.G;
  int lo = 0, hi = a.tk, len = a.tk;
  if (a.lens) len = hi = max(0, min(a.lens[b], a.tk));
  if (a.spans) {
    const int2 s = a.spans[(size_t)b * a.tq + t];
    lo = max(s.x, 0);
    hi = min(s.y, a.tk);
  } else if (a.causal) {
    hi = (int)min((long long)a.tk, max(0ll, (long long)a.q_start + t + 1));
  }
  const int pos = a.pos ? a.pos[(size_t)b * a.tq + t] : a.pos_at_len ? len : a.q_start + t;
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  s_q[tid] = load16<F16>(a.q, b * a.q_b + h * a.q_h + t * a.q_t + tid);
  float m = -INFINITY, l = 0.f, o = 0.f;
  __syncthreads();
  for (int j0 = lo; j0 < hi; j0 += 128) {
    const int j = j0 + tid;
    float s = -INFINITY;
    if (j < hi) {
      float acc = 0.f;
      const long long base = b * a.k_b + kv * a.k_h + (long long)j * a.k_t;
      for (int c = 0; c < 128; ++c) acc = fmaf(s_q[c], load16<F16>(a.k, base + c), acc);
      s = acc * a.sm_scale;
      if (a.softcap > 0.f) s = a.softcap * tanhf(s / a.softcap);
      s -= slope * fabsf((float)(pos - j));
    }
    float mx = s;
    for (int off = 16; off; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
    if ((tid & 31) == 0) s_red[tid >> 5] = mx;
    __syncthreads();
    const float mn = fmaxf(m, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float p = j < hi ? expf(s - ref) : 0.f;
    s_p[tid] = p;
    const float c = m == -INFINITY ? 0.f : expf(m - ref);
    m = mn;
    __syncthreads();
    float sum = 0.f, acc = 0.f;
    const int n = min(128, hi - j0);
    const long long base = b * a.v_b + kv * a.v_h + (long long)j0 * a.v_t + tid;
    for (int i = 0; i < n; ++i) {
      sum += s_p[i];
      acc = fmaf(s_p[i], load16<F16>(a.v, base + i * a.v_t), acc);
    }
    l = l * c + sum;
    o = o * c + acc;
    __syncthreads();
  }
  float lse = l == 0.f ? -INFINITY : m + logf(l);
  float r = l == 0.f ? 0.f : o / l;
  if (a.own_out) {
    const size_t row = ((size_t)b * a.tq + t) * a.heads_q + h;
    const float om = a.own_ml[2 * row], ol = a.own_ml[2 * row + 1];
    const float mine = ol == 0.f ? -INFINITY : om + logf(ol);
    const float top = fmaxf(lse, mine);
    if (mine != -INFINITY) {
      const float w0 = expf(lse - top), w1 = expf(mine - top);
      r = (r * w0 + a.own_out[row * 128 + tid] * w1) / (w0 + w1);
      lse = top + logf(w0 + w1);
    }
  }
  const long long at = b * a.o_b + h * a.o_h + t * a.o_t + tid;
  if (OUT32)
    static_cast<float*>(a.out)[at] = r;
  else if (F16)
    static_cast<__half*>(a.out)[at] = __float2half_rn(r);
  else
    static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(r);
  if (a.stat && tid == 0) {
    const long long i = b * a.s_b + h * a.s_h + t * a.s_t;
    if (a.stat_pair) {
      a.stat[2 * i] = lse;
      a.stat[2 * i + 1] = lse == -INFINITY ? 0.f : 1.f;
    } else {
      a.stat[i] = lse;
    }
  }
}

}  // namespace

size_t flash_workspace_bytes(int, int, int, int, int, int) { return kWsHeader; }

cudaError_t launch_flash(const FlashArgs& a, bool f16, bool out_f32, void*, int, cudaStream_t st) {
  auto k = f16 ? (out_f32 ? flash_rows_kernel<true, true> : flash_rows_kernel<true, false>)
               : (out_f32 ? flash_rows_kernel<false, true> : flash_rows_kernel<false, false>);
  k<<<dim3(a.tq, a.heads_q, a.batch), 128, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace mikv
