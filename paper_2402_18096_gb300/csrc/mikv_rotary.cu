// mikv_rotary.cu — rotary positions and the visible-key spans of a prompt (sm_103a).
//
// Rotary: a pair of channels (x, x') of a token at position p turns by a = 2 pi p f (f: turns per position). The
// product p f is formed modulo one turn in 64-bit integer arithmetic (f as a 64-bit fraction), where a 32-bit float
// product would lose 2^-24 of the whole angle. The angle is off by at most |p| 2^-55 turns (the fraction comes from doubles:
// frequencies up to 1 radian per position), 2^-32 (the bits kept) and 2^-26 (their rounding to fp32).
// Bound by HBM: every element is read and written once. A block takes a few tokens of some heads, at most four 32-byte
// items to a thread: the loads are issued first, the cosines and sines of the block's tokens are computed while
// they are under way (once, in shared memory, for all heads), then everything is turned and written.
#include "mikv_device.cuh"
#include "mikv_internal.h"
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

constexpr int kRotItems = 4;  // items of a thread

// cos and sin of the block's tokens, [tokens][rot / 2]
__device__ __forceinline__ void rotary_angles(const RotaryArgs& a, float2* cs, int b, int t0, int nt) {
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < nt * half; i += kRotThreads) {
    const int t = i / half, f = i - t * half;
    const long long pos = a.positions ? a.positions[(size_t)b * a.tokens + t0 + t] : (long long)a.start + t0 + t;
    const unsigned long long turn = (unsigned long long)pos * a.phases[f];  // modulo 2^64 = one turn
    float s, c;
    sincospif((float)(int)(turn >> 32) * 0x1p-31f, &s, &c);
    cs[i] = make_float2(c * a.amplitude, (a.inverse ? -s : s) * a.amplitude);
  }
}

// Rows of 16-byte vectors: an item is two of them. HALF: a vector of the first turning half with its partner, or two
// copied ones (the number of copied vectors is even: rot / 2 is a whole number of vectors and so is d / 2).
// Interleaved: two neighbours. A thread keeps its token and its place in the row and takes several heads, so that it
// reads its angles from shared memory once; a warp has one token, so that those reads meet in few banks.
// log_tok: log2 of the tokens of a block; heads [z * heads_z, ...) of both tensors.
template <typename T, bool HALF>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const __grid_constant__ RotaryArgs a, int log_tok, int heads_z) {
  extern __shared__ float2 s_cs[];
  constexpr int N = Vec<T>::N, kPerRow = kHeadDim / N / 2;
  const int half = a.rot / 2, b = blockIdx.y, t0 = blockIdx.x << log_tok, nt = min(1 << log_tok, a.tokens - t0);
  const int h0 = blockIdx.z * heads_z, nh = min(heads_z, a.x[0].heads + a.x[1].heads - h0);
  const int per_tok = kRotThreads >> log_tok, t = threadIdx.x / per_tok, r = threadIdx.x - t * per_tok;
  const int it = r % kPerRow, step = per_tok / kPerRow;
  const int turning = half / N;
  const int ch = !HALF ? 2 * it * N : it < turning ? it * N : a.rot + (it - turning) * N;
  const int gap = !HALF ? N : ch < a.rot ? half : (kHeadDim - a.rot) / 2;
  Vec<T> lo[kRotItems], hi[kRotItems];
  T* out[kRotItems];
  grid_dependency_wait();
  allow_dependent_launch();
#pragma unroll
  for (int u = 0; u < kRotItems; ++u) {
    const int hz = r / kPerRow + u * step;
    out[u] = nullptr;
    if (t >= nt || hz >= nh) continue;
    const bool second = h0 + hz >= a.x[0].heads;
    const int h = h0 + hz - (second ? a.x[0].heads : 0);
    const RotaryTensor& x = second ? a.x[1] : a.x[0];
    const T* in = static_cast<const T*>(x.in) + b * x.in_b + h * x.in_h + (t0 + t) * x.in_t + ch;
    out[u] = static_cast<T*>(x.out) + b * x.out_b + h * x.out_h + (t0 + t) * x.out_t + ch;
    lo[u].u = *reinterpret_cast<const uint4*>(in);
    hi[u].u = *reinterpret_cast<const uint4*>(in + gap);
  }
  rotary_angles(a, s_cs, b, t0, nt);
  __syncthreads();
  // N pairs: of the two vectors' channels (HALF), or N / 2 of each vector
  float2 w[N];
  const float2* cs = s_cs + t * half + (HALF ? ch : ch / 2);
  const bool turn0 = t < nt && ch < a.rot, turn1 = HALF ? turn0 : t < nt && ch + N < a.rot;
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (HALF || e < N / 2 ? turn0 : turn1) w[e] = cs[e];
#pragma unroll
  for (int u = 0; u < kRotItems; ++u) {
    if (!out[u]) continue;
    if constexpr (HALF) {
      if (turn0) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float p = to_f32(lo[u].e[e]), q = to_f32(hi[u].e[e]);
          lo[u].e[e] = from_f32<T>(p * w[e].x - q * w[e].y);
          hi[u].e[e] = from_f32<T>(p * w[e].y + q * w[e].x);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        Vec<T>& x = v ? hi[u] : lo[u];
        if (v ? turn1 : turn0) {
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const float2 c = w[(v * N + e) / 2];
            const float p = to_f32(x.e[e]), q = to_f32(x.e[e + 1]);
            x.e[e] = from_f32<T>(p * c.x - q * c.y);
            x.e[e + 1] = from_f32<T>(p * c.y + q * c.x);
          }
        }
      }
    }
    *reinterpret_cast<uint4*>(out[u]) = lo[u].u;
    *reinterpret_cast<uint4*>(out[u] + gap) = hi[u].u;
  }
}

// Any alignment, strides and number of turning channels: a pair or a copied channel at a time. Bound by instructions (two
// divisions and two 2- or 4-byte accesses each way per pair): 8192 tokens of 40 heads in rows of 131 elements take 124 us
// in bf16 (1.4 TB/s, 20 % of a copy) and 132 in fp32 (38 %), with 10 turning channels 197 and 218; aligned 27 and 51 us in
// rotary_kernel. Whole models have aligned rows; this form is there so that no view is refused.
template <typename T, bool HALF>
__global__ void __launch_bounds__(kRotThreads) rotary_elements_kernel(const __grid_constant__ RotaryArgs a, int log_tok) {
  extern __shared__ float2 s_cs[];
  const int half = a.rot / 2, b = blockIdx.y, t0 = blockIdx.x << log_tok, nt = min(1 << log_tok, a.tokens - t0);
  grid_dependency_wait();
  allow_dependent_launch();
  rotary_angles(a, s_cs, b, t0, nt);
  __syncthreads();
  const int items = half + kHeadDim - a.rot;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const RotaryTensor& x = a.x[which];
    const int per_tok = x.heads * items;
    for (int i = threadIdx.x; i < nt * per_tok; i += kRotThreads) {
      const int t = i / per_tok, r = i - t * per_tok;
      const int h = r / items, it = r - h * items;
      const T* in = static_cast<const T*>(x.in) + b * x.in_b + h * x.in_h + (t0 + t) * x.in_t;
      T* out = static_cast<T*>(x.out) + b * x.out_b + h * x.out_h + (t0 + t) * x.out_t;
      if (it >= half) {  // copied channels
        out[a.rot + it - half] = in[a.rot + it - half];
        continue;
      }
      const int c0 = HALF ? it : 2 * it, c1 = HALF ? it + half : 2 * it + 1;
      const float2 w = s_cs[t * half + it];
      const float p = to_f32(in[c0]), q = to_f32(in[c1]);
      out[c0] = from_f32<T>(p * w.x - q * w.y);
      out[c1] = from_f32<T>(p * w.y + q * w.x);
    }
  }
}

template <typename T>
cudaError_t launch_rotary_t(const RotaryArgs& a, int layout, bool vec, cudaStream_t st) {
  // Eight tokens to a block write each head's rows 2 KB at a time: 32768 tokens of 32 + 8 bf16 heads take 97 us in a graph (104
  // call by call, 95 % of a copy), 100 with two or four tokens, 135 with one (which also computes each angle for fewer
  // heads). Few tokens are spread over more blocks instead (one / eight tokens to a block): 128 tokens of 32 + 8 bf16 heads
  // 2.0 / 2.7 us, of 40 + 40 fp32 heads 2.8 / 3.4; 2048 tokens 11.0 / 9.1 and 25.8 / 26.6. Between, 512 and 1024 tokens of
  // 32 + 8 bf16 heads would gain from eight (4.4 / 3.6, 7.0 / 5.6), fp32 would lose (4.9 / 5.8, 8.1 / 8.1).
  const int log_tok = a.tokens >= 8 && (long long)a.batch * a.tokens >= 2048 ? 3 : 0, tok = 1 << log_tok;
  const int blocks = (a.tokens + tok - 1) / tok;
  const size_t smem = (size_t)tok * (a.rot / 2) * sizeof(float2);
  if (!vec) {
    auto k = layout == 0 ? rotary_elements_kernel<T, true> : rotary_elements_kernel<T, false>;
    return launch_chained(k, dim3(blocks, a.batch), dim3(kRotThreads), smem, st, a, log_tok);
  }
  const int heads = a.x[0].heads + a.x[1].heads;
  const int most = kRotThreads * kRotItems / (kHeadDim / Vec<T>::N / 2) / tok;  // heads of a block
  const int parts = (heads + most - 1) / most;
  if (parts > 65535) return cudaErrorInvalidValue;
  auto k = layout == 0 ? rotary_kernel<T, true> : rotary_kernel<T, false>;
  return launch_chained(k, dim3(blocks, a.batch, parts), dim3(kRotThreads), smem, st, a, log_tok,
                        (heads + parts - 1) / parts);
}

// One thread per query: the document that holds its position by binary search.
__global__ void __launch_bounds__(256) mask_spans_kernel(const SpanArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
  grid_dependency_wait();
  allow_dependent_launch();
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
  return launch_chained(mask_spans_kernel, dim3((a.tq + 255) / 256, a.batch), dim3(256), 0, st, a);
}

}  // namespace mikv
