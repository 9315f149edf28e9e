// mikv_rotary.cu — rotary positions and the visible-key spans of a prompt (sm_103a).
//
// Rotary: a pair of channels (x, x') of a token at position p turns by a = 2 pi p f (f: turns per position). The
// product p f is formed modulo one turn in 64-bit integer arithmetic (f as a 64-bit fraction), so its error stays
// below 2^-32 turns at any position, where a 32-bit float product would lose 2^-24 of the whole angle. Each block
// computes the cosines and sines of its tokens once, in shared memory, for all heads of both tensors.
// Bound by HBM: every element is read and written once.
#include "mikv_device.cuh"
#include "mikv_rotary.h"

namespace mikv {
namespace {

constexpr int kRotThreads = 256;

template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float to_f32(float x) { return x; }

template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ float from_f32(float x) { return x; }

// 16 bytes of elements.
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  union {
    uint4 u;
    T e[N];
  };
};

// Items of one head row, in elements: VEC: vectors of 16 bytes (HALF: one from each half of the turning channels per
// item); scalar: one pair per item. Channels past `rot` are copied, one vector / one element per item.
template <typename T, bool HALF, bool VEC>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const __grid_constant__ RotaryArgs a, int tok_per_block) {
  extern __shared__ float2 s_cs[];  // [tok_per_block][rot / 2] (cos, sin)
  constexpr int N = VEC ? Vec<T>::N : 1;
  const int half = a.rot / 2;
  const int b = blockIdx.y;
  const int t0 = blockIdx.x * tok_per_block;
  const int nt = min(tok_per_block, a.tokens - t0);
  for (int i = threadIdx.x; i < nt * half; i += kRotThreads) {
    const int t = i / half, f = i - t * half;
    const long long pos = a.positions ? a.positions[(size_t)b * a.tokens + t0 + t] : (long long)a.start + t0 + t;
    const unsigned long long turn = (unsigned long long)pos * a.phases[f];  // modulo 2^64 = one turn
    float s, c;
    sincospif((float)(int)(turn >> 32) * 0x1p-31f, &s, &c);
    s_cs[i] = make_float2(c * a.amplitude, (a.inverse ? -s : s) * a.amplitude);
  }
  __syncthreads();
  const int turning = HALF ? half / N : (VEC ? a.rot / N : half);
  const int items = turning + (kHeadDim - a.rot) / N;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const RotaryTensor& x = a.x[which];
    const int per_tok = x.heads * items;
    for (int i = threadIdx.x; i < nt * per_tok; i += kRotThreads) {
      const int t = i / per_tok, r = i - t * per_tok;
      const int h = r / items, it = r - h * items;
      const T* in = static_cast<const T*>(x.in) + b * x.in_b + h * x.in_h + (t0 + t) * x.in_t;
      T* out = static_cast<T*>(x.out) + b * x.out_b + h * x.out_h + (t0 + t) * x.out_t;
      const float2* cs = s_cs + t * half;
      if (it >= turning) {  // copied channels
        const int c0 = a.rot + (it - turning) * N;
        if constexpr (VEC)
          *reinterpret_cast<uint4*>(out + c0) = *reinterpret_cast<const uint4*>(in + c0);
        else
          out[c0] = in[c0];
        continue;
      }
      if constexpr (VEC && HALF) {
        Vec<T> lo, hi;
        lo.u = *reinterpret_cast<const uint4*>(in + it * N);
        hi.u = *reinterpret_cast<const uint4*>(in + half + it * N);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 w = cs[it * N + e];
          const float p = to_f32(lo.e[e]), q = to_f32(hi.e[e]);
          lo.e[e] = from_f32<T>(p * w.x - q * w.y);
          hi.e[e] = from_f32<T>(p * w.y + q * w.x);
        }
        *reinterpret_cast<uint4*>(out + it * N) = lo.u;
        *reinterpret_cast<uint4*>(out + half + it * N) = hi.u;
      } else if constexpr (VEC) {
        Vec<T> v;
        v.u = *reinterpret_cast<const uint4*>(in + it * N);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const float2 w = cs[(it * N + e) / 2];
          const float p = to_f32(v.e[e]), q = to_f32(v.e[e + 1]);
          v.e[e] = from_f32<T>(p * w.x - q * w.y);
          v.e[e + 1] = from_f32<T>(p * w.y + q * w.x);
        }
        *reinterpret_cast<uint4*>(out + it * N) = v.u;
      } else {
        const int c0 = HALF ? it : 2 * it, c1 = HALF ? it + half : 2 * it + 1;
        const float2 w = cs[it];
        const float p = to_f32(in[c0]), q = to_f32(in[c1]);
        out[c0] = from_f32<T>(p * w.x - q * w.y);
        out[c1] = from_f32<T>(p * w.y + q * w.x);
      }
    }
  }
}

template <typename T>
cudaError_t launch_rotary_t(const RotaryArgs& a, int layout, bool vec, cudaStream_t st) {
  const int tok = a.tokens >= 4 ? 4 : 1;
  const dim3 grid((a.tokens + tok - 1) / tok, a.batch);
  const size_t smem = (size_t)tok * (a.rot / 2) * sizeof(float2);
  auto k = layout == 0 ? (vec ? rotary_kernel<T, true, true> : rotary_kernel<T, true, false>)
                       : (vec ? rotary_kernel<T, false, true> : rotary_kernel<T, false, false>);
  k<<<grid, kRotThreads, smem, st>>>(a, tok);
  return cudaGetLastError();
}

// One thread per query: the document that holds its position by binary search.
__global__ void __launch_bounds__(256) mask_spans_kernel(const SpanArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
  if (i >= a.tq) return;
  const long long p = (long long)a.q_start + i;
  long long lo = 0, hi = a.causal ? p + 1 : a.tk;
  int doc = 0;
  bool none = false;
  long long doc_end = a.tk;
  if (a.docs) {
    const int32_t* off = a.docs + (size_t)b * (a.n_docs + 1);
    int l = 0, r = a.n_docs + 1;  // the number of offsets <= p
    while (l < r) {
      const int m = (l + r) >> 1;
      if (off[m] <= p)
        l = m + 1;
      else
        r = m;
    }
    none = l == 0 || l > a.n_docs;
    doc = none ? 0 : l - 1;
    lo = off[doc];
    doc_end = off[doc + 1];
  }
  if (a.prefix) hi = max(hi, lo + a.prefix[(size_t)b * (a.docs ? a.n_docs : 1) + doc]);
  hi = min(hi, min(doc_end, (long long)a.tk));
  if (a.key_len) hi = min(hi, (long long)a.key_len[b]);
  lo = max(lo, 0ll);
  if (none || hi <= lo) lo = hi = 0;
  a.spans[(size_t)b * a.tq + i] = make_int2((int)lo, (int)hi);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, int dtype, int layout, bool vec, cudaStream_t st) {
  if (dtype == 0) return launch_rotary_t<__nv_bfloat16>(a, layout, vec, st);
  if (dtype == 1) return launch_rotary_t<__half>(a, layout, vec, st);
  return launch_rotary_t<float>(a, layout, vec, st);
}

cudaError_t launch_mask_spans(const SpanArgs& a, cudaStream_t st) {
  mask_spans_kernel<<<dim3((a.tq + 255) / 256, a.batch), 256, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace mikv
