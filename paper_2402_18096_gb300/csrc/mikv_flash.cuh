// mikv_flash.cuh — attention over bf16 / fp16 keys on the fifth-generation tensor cores (sm_103a): the kernel
// template of the prompt and shared-prefix entry points. mikv_flash_bf16.cu and mikv_flash_f16.cu instantiate it for
// one operand type each; mikv_flash.cu holds the work plan, the merge of split parts and the dispatch.
//
// Problem. `batch` sets of keys; each set is attended by tq tokens of G query heads per KV head (a prompt's tokens are
// its positions, a shared prefix's tokens are its requests). The tq * G query rows of one KV head are packed into
// tiles of 128 rows, row R = token * G + head, so that all heads and tokens that share keys share their loads.
//
// One CTA works on two streams, each with a score tile S (128 x 128 fp32) and an output tile O (128 x 128 fp32) in
// TMEM, over 128-key tiles of K and V that TMA stages in a ring:
//   PAIR    two row tiles (256 rows) over the same key tiles: a K or V tile is loaded once for both.
//   !PAIR   one row tile (up to 128 rows) over alternating key tiles; the streams' results are joined at the end.
//           The second stream's loads and softmax overlap the first's, which keeps HBM busy when rows are few.
// Roles: warps 0-3 and 4-7 are the streams' softmax warpgroups (thread = row = TMEM lane), warp 8 issues the copies,
// warp 9 the MMAs, warps 10-11 guard masked tiles (below). Per stream and tile: S = Q K^T (8 MMAs of K = 16), softmax
// to P (16-bit, written over S in TMEM), O += P V (8 MMAs with A in TMEM). The MMA warp alternates streams, so one
// stream's softmax runs under the other's products.
//
// Softmax. Weights are 2^(x - r) with x the score in log2 units and r a reference of the row: the largest x of the
// first tile the row sees (less kRefDrop), moved only when a tile's sum of weights passes kSumMax, which rescales O. The
// weights' 16-bit types hold that range without loss of relative precision, so most tiles need no maximum at all. Key
// tiles are visited from the last to the first: with a causal mask or a distance bias the largest scores then
// tend to come first. Sums are fp32 over the unrounded weights; rounding the weights to 16 bits is what the tensor
// cores take, and perturbs each weight by at most half a unit in its last place.
//
// Masks. Every row sees one span of keys [lo, hi). Tiles outside the union of the CTA's spans are not visited; tiles
// inside every span are not masked. In the tiles between, a weight of 0 does not stop an infinity or NaN in V from
// entering O (0 * inf), so the guard warps look through the V tile first: rows with such a value are set to 0 and
// their keys reported to the softmax threads, which mark the output rows that do see them.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <limits.h>
#include <math.h>

#include <atomic>

#include "mikv_device.cuh"
#include "mikv_flash.h"
#include "mikv_tcgen05.cuh"

namespace mikv {

template <bool F16>
cudaError_t launch_flash_kernel(const FlashKernelArgs& p, bool pair, dim3 grid, cudaStream_t st);

namespace flash {

constexpr int kTile = 128;                     // query rows of a tile, keys of a tile
constexpr int kTileBytes = kTile * kHeadDim * 2;
constexpr int kHalfBytes = kTileBytes / 2;     // one 64-channel box
constexpr int kSoftThreads = 256;
constexpr int kCopyWarp = 8, kMmaWarp = 9, kGuardWarp = 10;
constexpr int kThreads = 384;
constexpr int kTmemCols = 512;                 // S0, S1, O0, O1
constexpr int kSafeRing = 4;                   // guard results in flight (more than V tiles of a stream in the ring)
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <bool PAIR>
struct Layout {
  static constexpr int kQ = PAIR ? 2 : 1;          // query tiles in shared memory
  static constexpr int kStages = PAIR ? 5 : 6;     // K / V tiles in the ring
  // Loads: the first kLead K tiles, then V tile u and K tile u + kLead for u = 0, 1, ... (from the last key tile on).
  static constexpr int kLead = PAIR ? 1 : 2;
  static constexpr int kBars = 1 + 2 * kStages + 5 * 2 + 2 * kSafeRing + 1;
  static constexpr int kSmem = 1024 + (kQ + kStages) * kTileBytes + 8 * kBars;
  static_assert(kSmem <= 227 * 1024, "shared memory of one CTA");
  uint32_t base;
  __device__ uint32_t q(int m) const { return base + m * kTileBytes; }
  __device__ uint32_t stage(int s) const { return base + (kQ + s) * kTileBytes; }
  __device__ uint32_t bar(int i) const { return base + (kQ + kStages) * kTileBytes + 8 * i; }
  __device__ uint32_t qfull() const { return bar(0); }
  __device__ uint32_t full(int s) const { return bar(1 + s); }               // a copy landed
  __device__ uint32_t empty(int s) const { return bar(1 + kStages + s); }    // it is not needed any more
  __device__ uint32_t sfull(int w) const { return bar(1 + 2 * kStages + w); }       // scores of stream w
  // of half a tile (64 keys): weights written (and O rescaled for them); O += P V done
  __device__ uint32_t pready(int w, int half) const { return bar(1 + 2 * kStages + 2 + 2 * w + half); }
  __device__ uint32_t odone(int w, int half) const { return bar(1 + 2 * kStages + 6 + 2 * w + half); }
  // guarded V tile looked through (PAIR: set 0 serves both streams)
  __device__ uint32_t vsafe(int w, int g) const { return bar(1 + 2 * kStages + 10 + kSafeRing * w + g % kSafeRing); }
  __device__ uint32_t drain() const { return bar(kBars - 1); }
};

// What the weights may grow to before the reference moves, and how far below a tile's largest score the reference is
// put (log2). bf16 weights have fp32's range, so the reference is that largest score and the sums may grow
// far; fp16 weights hold 2^-24 .. 2^16, so they start at 2^8 and move before the sum of a tile can pass 2^16.
template <bool F16>
__device__ constexpr float ref_drop() { return F16 ? 8.f : 0.f; }
template <bool F16>
__device__ constexpr float sum_max() { return F16 ? 0x1.fep15f : 0x1p20f; }
// A largest score this far above the reference may stay: 128 weights of 2^it are below sum_max.
template <bool F16>
__device__ constexpr float ref_slack() { return F16 ? 8.5f : 12.f; }

// Above this size of the reference, scores are rounded before it is taken off (the slow path): the fused form keeps
// the product's rounding error, up to 2^-24 of it, which would be a factor of the weights.
constexpr float kRefExact = 0x1p22f;

// The scores of one row in log2 units: x = cap(v * scale) - slope |pos - j|, times log2 e.
struct Row {
  int lo, hi;        // keys the row sees
  float pos;         // its position, as far as the bias needs it (exact below 2^24)
  float slope;       // slope of its head times log2 e
};

struct Score {
  float scale;     // uncapped: sm_scale log2 e; capped: 2 log2 e sm_scale / cap
  float cap;       // cap log2 e
};

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {  // NaN if either is
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// The cap of four scores: cap tanh(y) + rest = (cap + rest) - 2 cap / (1 + e^2y). One reciprocal serves all four:
// with p = (ac, bd) of the denominators a, b, c, d, 1 / a = bd c / (ac bd) and so on. 2^30 stands for larger
// exponentials (tanh is then 1 to fp32 precision), which keeps the product of four inside fp32.
__device__ __forceinline__ void cap_four(float* v, float scale, float cap, const float (&rest)[4]) {
  const uint64_t s2 = f32x2(scale, scale), one = f32x2(1.f, 1.f), c2 = f32x2(-2.f * cap, -2.f * cap);
  float y[4];
  f32x2_split(mul_f32x2(f32x2(v[0], v[1]), s2), y[0], y[1]);
  f32x2_split(mul_f32x2(f32x2(v[2], v[3]), s2), y[2], y[3]);
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = fast_exp2(min_nan(y[i], 30.f));
  const uint64_t ab = add_f32x2(f32x2(y[0], y[1]), one), cd = add_f32x2(f32x2(y[2], y[3]), one);
  float ac, bd;
  f32x2_split(mul_f32x2(ab, cd), ac, bd);
  const float r = rcp_approx(ac * bd);
  const uint64_t s = mul_f32x2(f32x2(r, r), f32x2(bd, ac));
  f32x2_split(fma_f32x2(mul_f32x2(s, cd), c2, f32x2(rest[0], rest[1])), v[0], v[1]);
  f32x2_split(fma_f32x2(mul_f32x2(s, ab), c2, f32x2(rest[2], rest[3])), v[2], v[3]);
}

__device__ __forceinline__ float max3(float a, float b, float c) {  // NaN operands are passed over
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// N scores (columns col0 .. of the tile at key k0) less `ref`, in place.
// side: every key of the tile lies at or before every position of the warp (-1), at or after them (1), or neither (0).
template <bool CAP, bool BIAS, int N>
__device__ __forceinline__ void row_scores(float* v, const Score& sc, const Row& row, int k0, int col0, float ref,
                                           int side) {
  const float rest = (CAP ? sc.cap : 0.f) - ref;
  auto apply = [&](auto bias) {  // bias(i): the bias of column i, plus `rest`
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float b[4] = {bias(i), bias(i + 1), bias(i + 2), bias(i + 3)};
      if constexpr (CAP) {
        cap_four(v + i, sc.scale, sc.cap, b);
      } else {
        const uint64_t s2 = f32x2(sc.scale, sc.scale);
        f32x2_split(fma_f32x2(f32x2(v[i], v[i + 1]), s2, f32x2(b[0], b[1])), v[i], v[i + 1]);
        f32x2_split(fma_f32x2(f32x2(v[i + 2], v[i + 3]), s2, f32x2(b[2], b[3])), v[i + 2], v[i + 3]);
      }
    }
  };
  if constexpr (!BIAS) {
    apply([&](int) { return rest; });
  } else {
    const float e0 = (float)(k0 + col0) - row.pos;
    if (side != 0) {  // the bias is linear over the tile
      const float sl = side < 0 ? row.slope : -row.slope;
      const float base = fmaf(sl, e0, rest);
      apply([&](int i) { return fmaf(sl, (float)i, base); });
    } else {
      apply([&](int i) { return fmaf(-row.slope, fabsf(e0 + (float)i), rest); });
    }
  }
}

// Scores outside the row's span, replaced by x.
template <int N>
__device__ __forceinline__ void mask_scores(float* v, const Row& row, int first_key, float x) {
  const int first = row.lo - first_key;
  const unsigned n = row.hi - row.lo;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if ((unsigned)(i - first) >= n) v[i] = x;
}

template <bool F16>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  return F16 ? pack_f16(a, b) : pack_bf16(a, b);
}

// Whether one of the eight 16-bit values is an infinity or NaN (its exponent bits all ones).
template <bool F16>
__device__ __forceinline__ bool any_nonfinite(const uint4& x) {
  constexpr uint32_t one = F16 ? 0x04000400u : 0x00800080u;  // carries into the sign bit from an all-ones exponent
  const uint32_t r = ((x.x & 0x7FFF7FFFu) + one) | ((x.y & 0x7FFF7FFFu) + one) | ((x.z & 0x7FFF7FFFu) + one) |
                     ((x.w & 0x7FFF7FFFu) + one);
  return (r & 0x80008000u) != 0;
}

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 r;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr)
               : "memory");
  return r;
}
__device__ __forceinline__ void sts128_zero(uint32_t addr) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(addr), "r"(0u) : "memory");
}

// S (128 x 128) = query tile x key tile^T.
template <bool F16>
__device__ __forceinline__ void mma_scores(uint32_t d, uint32_t q, uint32_t k) {
  constexpr uint32_t idesc = umma_idesc_16(F16, kTile, kTile, false);
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    const uint32_t off = (ks >> 2) * kHalfBytes + (ks & 3) * 32;
    umma_bf16(d, umma_desc_sw128(q + off), umma_desc_sw128(k + off), idesc, ks > 0 ? 1u : 0u);
  }
}

// O (128 x 128) += P (TMEM, 128 x 128) x V tile, 64 of the keys.
template <bool F16>
__device__ __forceinline__ void mma_values(uint32_t d, uint32_t p, uint32_t v, int half, bool accumulate) {
  constexpr uint32_t idesc = umma_idesc_16(F16, kTile, kTile, true);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int ks = 4 * half + i;
    umma_16_ts(d, p + 8 * ks, umma_desc_rows_sw128(v + ks * 16 * 128, kHalfBytes), idesc,
               (ks > 0 || accumulate) ? 1u : 0u);
  }
}

// Four packed outputs at element i of an output row (16-byte stores for a caller that walks 8 / 4 elements).
__device__ __forceinline__ void store_out8(void* row, int out_kind, int i, const float* v) {
  if (out_kind == 2) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(row) + i);
    o[0] = make_float4(v[0], v[1], v[2], v[3]);
    o[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else if (out_kind == 1) {
    *reinterpret_cast<uint4*>(static_cast<__half*>(row) + i) =
        make_uint4(pack_f16(v[0], v[1]), pack_f16(v[2], v[3]), pack_f16(v[4], v[5]), pack_f16(v[6], v[7]));
  } else {
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(row) + i) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
}

__device__ __forceinline__ void store_stat(const FlashArgs& a, long long i, float lse2) {
  if (!a.stat) return;
  if (a.stat_pair) {
    a.stat[2 * i] = lse2 * kLn2;
    a.stat[2 * i + 1] = lse2 == -INFINITY ? 0.f : 1.f;
  } else {
    a.stat[i] = lse2 * kLn2;
  }
}

// Join of a part (log2 of its sum: lse2) with the request's own part: factors of both outputs, and the joint lse2.
__device__ __forceinline__ void join_own(const FlashArgs& a, size_t row, float& lse2, float& f0, float& f1) {
  const float m = a.own_ml[2 * row], l = a.own_ml[2 * row + 1];
  const float mine = l == 0.f ? -INFINITY : fmaf(m, kLog2e, log2f(l));
  f1 = 0.f;
  if (mine == -INFINITY) return;
  const float top = fmaxf(lse2, mine);
  const float w0 = fast_exp2(lse2 - top), w1 = fast_exp2(mine - top), inv = 1.f / (w0 + w1);
  f0 *= w0 * inv;
  f1 = w1 * inv;
  lse2 = top + log2f(w0 + w1);
}

template <bool F16, bool PAIR, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) flash_kernel(const __grid_constant__ FlashKernelArgs p) {
  using L = Layout<PAIR>;
  const FlashArgs& a = p.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;
  __shared__ int s_range[8][4];
  __shared__ uint32_t s_bad[2][kSafeRing][4];  // keys of a guarded V tile that hold infinities or NaN
  volatile int* fail = &s_fail;
  L sm;
  sm.base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int h = blockIdx.y, b = blockIdx.z;
  const int split = blockIdx.x % p.n_splits;
  const int m_blocks = gridDim.x / p.n_splits;
  const int m_block = m_blocks - 1 - (int)(blockIdx.x / p.n_splits);  // a causal prompt's longest rows first

  if (tid == 0) {
    s_fail = 0;
    mbar_init(sm.qfull(), 1);
    for (int s = 0; s < L::kStages; ++s) {
      mbar_init(sm.full(s), 1);
      mbar_init(sm.empty(s), 3);  // its MMAs, and both guard warps
    }
    for (int w = 0; w < 2; ++w) {
      mbar_init(sm.sfull(w), 1);
      mbar_init(sm.pready(w, 0), 4);  // one arrival per softmax warp
      mbar_init(sm.pready(w, 1), 4);
      mbar_init(sm.odone(w, 0), 1);
      mbar_init(sm.odone(w, 1), 1);
    }
    for (int u = 0; u < 2 * kSafeRing; ++u) mbar_init(sm.vsafe(u / kSafeRing, u % kSafeRing), 2);
    mbar_init(sm.drain(), 1);
    fence_mbar_init();
  }
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&s_tmem), kTmemCols);
  if (p.n_splits > 1) allow_dependent_launch();  // the merge may be scheduled; it waits for this grid's end

  // this thread's row (softmax threads), and what the rows of each tile see
  const int stream = (warp >> 2) & 1, r = tid & (kTile - 1);
  const int R = (PAIR ? (2 * m_block + stream) : m_block) * kTile + r;
  const int token = R / a.G, head = h * a.G + R % a.G;
  const bool valid = warp < kCopyWarp && token < a.tq;
  Row row;
  row.lo = row.hi = 0;
  row.pos = 0.f;
  row.slope = 0.f;
  int warp_lo = INT_MAX, warp_hi = 0, warp_all_lo = 0, warp_all_hi = 0, pos_min = 0, pos_max = 0;
  if (warp < kCopyWarp) {
    int at = 0;
    if (valid) {
      int len = a.tk;
      row.hi = a.tk;
      if (a.lens) len = row.hi = max(0, min(a.lens[b], a.tk));
      if (a.spans) {
        const int2 s = a.spans[(size_t)b * a.tq + token];
        row.lo = max(s.x, 0);
        row.hi = min(s.y, a.tk);
      } else if (a.causal) {
        row.hi = (int)min((long long)a.tk, max(0ll, (long long)a.q_start + token + 1));
      }
      if constexpr (BIAS) {
        at = a.pos ? a.pos[(size_t)b * a.tq + token] : a.pos_at_len ? len : a.q_start + token;
        row.pos = (float)at;
        row.slope = a.slopes[head] * kLog2e;
      }
      if (row.hi <= row.lo) row.lo = row.hi = 0;
    }
    const bool sees = row.hi > row.lo;
    warp_lo = __reduce_min_sync(0xffffffffu, sees ? row.lo : INT_MAX);
    warp_hi = __reduce_max_sync(0xffffffffu, row.hi);
    warp_all_lo = __reduce_max_sync(0xffffffffu, !valid ? 0 : sees ? row.lo : INT_MAX);
    warp_all_hi = __reduce_min_sync(0xffffffffu, !valid ? INT_MAX : row.hi);
    if (BIAS) {
      pos_min = __reduce_min_sync(0xffffffffu, valid ? at : INT_MAX);
      pos_max = __reduce_max_sync(0xffffffffu, valid ? at : INT_MIN);
    }
    if (lane == 0) {
      s_range[warp][0] = warp_lo;
      s_range[warp][1] = warp_hi;
      s_range[warp][2] = warp_all_lo;
      s_range[warp][3] = warp_all_hi;
    }
  }
  tcgen05_before_sync();
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = s_tmem;
  // per stream: key tiles [t0, t1) that some row sees, keys [all_lo, all_hi) that every row sees
  int t0[2], t1[2], all_lo[2], all_hi[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int lo = INT_MAX, hi = 0;
    all_lo[w] = 0;
    all_hi[w] = INT_MAX;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo = min(lo, s_range[4 * w + i][0]);
      hi = max(hi, s_range[4 * w + i][1]);
      all_lo[w] = max(all_lo[w], s_range[4 * w + i][2]);
      all_hi[w] = min(all_hi[w], s_range[4 * w + i][3]);
    }
    t0[w] = __shfl_sync(0xffffffffu, hi > 0 ? lo / kTile : INT_MAX, 0);  // (the same in every lane: a uniform value)
    t1[w] = __shfl_sync(0xffffffffu, (hi + kTile - 1) / kTile, 0);
    all_lo[w] = __shfl_sync(0xffffffffu, all_lo[w], 0);
    all_hi[w] = __shfl_sync(0xffffffffu, all_hi[w], 0);
  }
  // this CTA's share of the union of both streams' tiles
  int T0 = min(t0[0], t0[1]), T1 = max(t1[0], t1[1]);
  if (T1 == 0) T0 = 0;
  if (p.n_splits > 1) {
    const int chunk = (T1 - T0 + p.n_splits - 1) / p.n_splits;
    T0 = min(T1, T0 + split * chunk);
    T1 = min(T1, T0 + chunk);
  }
  const int n = T1 - T0;
  const int n_w[2] = {(n + 1) / 2, n / 2};  // !PAIR: tiles of each stream
  auto of = [](const int(&x)[2], int w) { return w ? x[1] : x[0]; };
  auto active = [&](int w, int j) { return j >= of(t0, w) && j < of(t1, w); };
  auto cut = [&](int w, int j) { return j * kTile < of(all_lo, w) || (j + 1) * kTile > of(all_hi, w); };
  auto guarded = [&](int j) { return PAIR ? (active(0, j) && cut(0, j)) || (active(1, j) && cut(1, j)) : cut(0, j); };

  // The softmax warps take the registers the other warpgroup does not need: 256 x 216 + 128 x 72 = 384 x 168.
  if (warp >= kCopyWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == kCopyWarp) {
      if (lane == 0 && n > 0) {
        int last[L::kStages];
        for (int s = 0; s < L::kStages; ++s) last[s] = -1;
        mbar_arrive_expect_tx(sm.qfull(), L::kQ * kTileBytes);
#pragma unroll
        for (int m = 0; m < L::kQ; ++m) {
          const int tok0 = (PAIR ? 2 * m_block + m : m_block) * (kTile / a.G);
          tma_load_4d(sm.q(m), &p.map_q, 0, h * a.G, tok0, b, sm.qfull());
          tma_load_4d(sm.q(m) + kHalfBytes, &p.map_q, 64, h * a.G, tok0, b, sm.qfull());
        }
        int c = 0;
        auto load = [&](const CUtensorMap* map, int j, int hm, int bm) {
          const int s = c % L::kStages;
          if (c >= L::kStages && !mbar_wait_role(sm.empty(s), ((c / L::kStages) & 1) ^ 1, fail)) return false;
          mbar_arrive_expect_tx(sm.full(s), kTileBytes);
          tma_load_4d(sm.stage(s), map, 0, j * kTile, h * hm, b * bm, sm.full(s));
          tma_load_4d(sm.stage(s) + kHalfBytes, map, 64, j * kTile, h * hm, b * bm, sm.full(s));
          last[s] = c++;
          return true;
        };
        auto load_k = [&](int j) { return load(&p.map_k, j, p.k_head, p.k_batch); };
        auto load_v = [&](int j) { return load(&p.map_v, j, p.v_head, p.v_batch); };
        bool ok = true;
        for (int u = 0; ok && u < min(n, L::kLead); ++u) ok = load_k(T1 - 1 - u);
        for (int u = 0; ok && u < n; ++u) ok = load_v(T1 - 1 - u) && (u + L::kLead >= n || load_k(T1 - 1 - u - L::kLead));
        // no copy may outlive the CTA, whatever became of the other roles
        if (!mbar_wait(sm.qfull(), 0)) record_error(a.status, kErrDrainTimeout);
        for (int s = 0; s < L::kStages; ++s)
          if (last[s] >= 0 && !mbar_wait(sm.full(s), (last[s] / L::kStages) & 1)) record_error(a.status, kErrDrainTimeout);
      }
    } else if (warp == kMmaWarp) {
      if (n > 0) {  // the whole warp, converged; one lane issues
        const bool leader = elect_one();
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        int done[2] = {0, 0};  // weights consumed per stream
        auto commit = [&](uint32_t bar) {
          if (leader) umma_commit(bar);
        };
        auto wait_full = [&](int c) {
          const bool ok = mbar_wait_warp(sm.full(c % L::kStages), (c / L::kStages) & 1, fail);
          tcgen05_after_sync();
          return ok;
        };
        auto scores = [&](int w, int c) {
          const uint32_t q = sm.q(PAIR ? w : 0), k = sm.stage(c % L::kStages);
          if (leader) {
            mma_scores<F16>(tm + 128 * w, q, k);
            umma_commit(sm.sfull(w));
          }
        };
        auto values = [&](int w, int c) {
          const uint32_t v = sm.stage(c % L::kStages);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (!mbar_wait_warp(sm.pready(w, half), of(done, w) & 1, fail)) return false;
            tcgen05_after_sync();
            if (leader) {
              mma_values<F16>(tm + 256 + 128 * w, tm + 128 * w, v, half, of(done, w) > 0);
              umma_commit(sm.odone(w, half));
            }
          }
          done[w ? 1 : 0] += 1;
          return true;
        };
        int checked[2] = {0, 0};  // guarded tiles so far (PAIR: in checked[0])
        auto wait_safe = [&](int w) {
          const int g = of(checked, w);
          checked[w ? 1 : 0] += 1;
          return mbar_wait_warp(sm.vsafe(w, g), (g / kSafeRing) & 1, fail);
        };
        bool ok = mbar_wait_warp(sm.qfull(), 0, fail) && wait_full(0);
        if constexpr (PAIR) {
          if (ok) {
#pragma unroll
            for (int w = 0; w < 2; ++w)
              if (active(w, T1 - 1)) scores(w, 0);
            commit(sm.empty(0));
          }
          for (int i = 0; ok && i < n; ++i) {
            const int j = T1 - 1 - i, cv = 2 * i + 1, ck = cv + 1;
            ok = wait_full(cv) && (!guarded(j) || wait_safe(0));
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              if (ok && active(w, j)) ok = values(w, cv);
              if (ok && i + 1 < n) {
                if (w == 0) ok = wait_full(ck);
                if (ok && active(w, j - 1)) scores(w, ck);
              }
            }
            if (ok) {
              commit(sm.empty(cv % L::kStages));
              if (i + 1 < n) commit(sm.empty(ck % L::kStages));
            }
          }
        } else {
          int c = 0;
#pragma unroll
          for (int w = 0; w < 2; ++w)
            if (ok && w < n) {
              if (w == 1) ok = wait_full(1);
              if (ok) {
                scores(w, c);
                commit(sm.empty(c));
                ++c;
              }
            }
          for (int i = 0; ok && i < of(n_w, 0); ++i) {
#pragma unroll
            for (int w = 0; w < 2; ++w)
              if (ok && i < of(n_w, w)) {
                ok = wait_full(c) && (!guarded(T1 - 1 - (2 * i + w)) || wait_safe(w)) && values(w, c);
                if (ok) {
                  commit(sm.empty(c % L::kStages));
                  ++c;
                }
                if (ok && i + 1 < of(n_w, w)) {
                  ok = wait_full(c);
                  if (ok) {
                    scores(w, c);
                    commit(sm.empty(c % L::kStages));
                    ++c;
                  }
                }
              }
          }
        }
        commit(sm.drain());  // every MMA issued has completed once this arrives
        if (!mbar_wait(sm.drain(), 0) && lane == 0) record_error(a.status, kErrDrainTimeout);
        __syncwarp();
      }
    } else {  // guard warps: they see every load in order and release it too (a wait that left out phases of a barrier
              // would take an earlier phase of the same parity for its own)
      int checked[2] = {0, 0}, c = 0;
      auto landed = [&]() { return mbar_wait_warp(sm.full(c % L::kStages), (c / L::kStages) & 1, fail); };
      auto release = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.empty(c % L::kStages));
        ++c;
      };
      bool ok = true;
      for (int u = 0; ok && u < min(n, L::kLead); ++u) {
        ok = landed();
        if (ok) release();
      }
      for (int u = 0; ok && u < n; ++u) {
        const int j = T1 - 1 - u, w = PAIR ? 0 : u & 1;
        ok = landed();
        if (!ok) break;
        if (guarded(j)) {
          const int g = of(checked, w);
          bool wrote = false;
#pragma unroll 1
          for (int part = warp - kGuardWarp; part < 4; part += 2) {
            const int key = 32 * part + lane;
            const uint32_t at = sm.stage(c % L::kStages) + key * 128;
            bool bad = false;
#pragma unroll
            for (int q = 0; q < 16; ++q)
              bad |= any_nonfinite<F16>(lds128(at + (q >> 3) * kHalfBytes + (((q & 7) ^ (key & 7)) << 4)));
            const uint32_t bits = __ballot_sync(0xffffffffu, bad);
            if (bad) {
              for (int q = 0; q < 16; ++q) sts128_zero(at + (q >> 3) * kHalfBytes + ((q & 7) << 4));
              wrote = true;
            }
            if (lane == 0) s_bad[w][g % kSafeRing][part] = bits;
          }
          if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(sm.vsafe(w, g));
          checked[w ? 1 : 0] += 1;
        }
        release();
        if (u + L::kLead < n) {
          ok = landed();
          if (ok) release();
        }
      }
    }
  } else {  // softmax warps
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t ts = tmem + 128 * stream + lanes, to = tmem + 256 + 128 * stream + lanes;
    Score sc;
    sc.scale = CAP ? 2.f * kLog2e * (a.sm_scale / a.softcap) : a.sm_scale * kLog2e;
    sc.cap = a.softcap * kLog2e;
    // (a row that sees nothing, or past the last token, needs no reference: its weights are 0 or never used)
    float ref = row.hi > row.lo ? -INFINITY : 0.f, sum = 0.f;
    bool bad_row = false, ok = true;
    bool careful = true;  // some row of the warp has no reference yet, or one beyond kRefExact
    const bool any_valid = __any_sync(0xffffffffu, valid);
    int it = 0, guards = 0;  // tiles done, guarded tiles met
    for (int i = 0; i < (PAIR ? n : of(n_w, stream)); ++i) {
      const int j = T1 - 1 - (PAIR ? i : 2 * i + stream);
      if (guarded(j)) ++guards;
      if (PAIR && !active(stream, j)) continue;
      const int k0 = j * kTile;
      ok = __all_sync(0xffffffffu, mbar_wait_role(sm.sfull(stream), it & 1, fail));
      if (!ok) break;
      tcgen05_after_sync();
      auto arrive = [&](int half) {
        tmem_wait_st();
        tcgen05_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.pready(stream, half));
      };
      if (k0 >= warp_hi || k0 + kTile <= warp_lo) {  // no row of this warp sees the tile
        if (any_valid) {  // (rows past the last token may hold anything)
          uint32_t zero[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) zero[e] = 0u;
          tmem_st32(ts, zero);
          tmem_st32(ts + 32, zero);
        }
        arrive(0);
        arrive(1);
        ++it;
        continue;
      }
      const bool masked = k0 < warp_all_lo || k0 + kTile > warp_all_hi;
      const int side = !BIAS ? 0 : k0 + kTile - 1 <= pos_min ? -1 : k0 >= pos_max ? 1 : 0;
      if (guarded(j)) {
        const int g = guards - 1, ws = PAIR ? 0 : stream;
        ok = __all_sync(0xffffffffu, mbar_wait_role(sm.vsafe(ws, g), (g / kSafeRing) & 1, fail));
        if (!ok) break;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t bits = s_bad[ws][g % kSafeRing][q];
          while (bits) {
            const int key = k0 + 32 * q + __ffs(bits) - 1;
            bits &= bits - 1;
            bad_row = bad_row || (key >= row.lo && key < row.hi);
          }
        }
      }
      // The weights of 64 columns, packed, and their sum: v holds the scores less the reference.
      auto pack_half = [&](const float (&v)[64], uint32_t (&w)[32]) {
        uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
        for (int e = 0; e < 64; e += 2) {
          const float x = fast_exp2(v[e]), y = fast_exp2(v[e + 1]);
          acc[(e >> 1) & 3] = add_f32x2(acc[(e >> 1) & 3], f32x2(x, y));
          w[e >> 1] = pack16<F16>(x, y);
        }
        float s0, s1, s2, s3;
        f32x2_split(add_f32x2(acc[0], acc[1]), s0, s1);
        f32x2_split(add_f32x2(acc[2], acc[3]), s2, s3);
        return (s0 + s1) + (s2 + s3);
      };
      auto load_half = [&](int half, float (&v)[64]) {
        tmem_ld32(ts + 64 * half, v);
        tmem_ld32(ts + 64 * half + 32, v + 32);
      };
      auto loaded = [](float (&v)[64]) {
        tmem_wait_ld(v);
        reg_fence(v + 32);
      };
      // Fast path: no mask, a reference in every row. Straight-line code for the whole tile, checked by the sum
      // afterwards; nothing is stored before the check.
      bool slow = masked || careful;
      if (!slow) {
        float v[2][64];
        uint32_t w[2][32];
        load_half(0, v[0]);
        loaded(v[0]);
        load_half(1, v[1]);
        row_scores<CAP, BIAS, 64>(v[0], sc, row, k0, 0, ref, side);
        float tile_sum = pack_half(v[0], w[0]);
        loaded(v[1]);
        row_scores<CAP, BIAS, 64>(v[1], sc, row, k0, 64, ref, side);
        tile_sum += pack_half(v[1], w[1]);
        slow = __any_sync(0xffffffffu, !(tile_sum <= sum_max<F16>()));  // a reference is too low (or a score NaN)
        if (!slow) {
          sum += tile_sum;
          tmem_st32(ts, w[0]);
          tmem_st32(ts + 32, w[1]);
          tmem_wait_st();
          tcgen05_before_sync();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(sm.pready(stream, 0));
            mbar_arrive(sm.pready(stream, 1));
          }
        }
      }
      // Slow path, 64 columns at a time: the largest score first, then the weights.
      if (slow) {
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          uint32_t w[32];
          float v[64];
          load_half(half, v);
          loaded(v);
          if (CAP && masked) mask_scores<64>(v, row, k0 + 64 * half, 0.f);  // (four share a reciprocal)
          row_scores<CAP, BIAS, 64>(v, sc, row, k0, 64 * half, 0.f, side);
          if (masked) mask_scores<64>(v, row, k0 + 64 * half, -INFINITY);
          float mx = -INFINITY, mx2 = -INFINITY;  // the row's largest score
#pragma unroll
          for (int e = 0; e < 64; e += 4) {
            mx = max3(mx, v[e], v[e + 1]);
            mx2 = max3(mx2, v[e + 2], v[e + 3]);
          }
          mx = fmaxf(mx, mx2);
          const float next = mx > ref + ref_slack<F16>() ? mx - ref_drop<F16>() : ref;
          const bool moves = next != ref && ref != -INFINITY;
          if (__any_sync(0xffffffffu, moves)) {
            const float f = moves ? fast_exp2(ref - next) : 1.f;
            if (it + half > 0) {  // O holds the products up to the half before this one
              ok = __all_sync(0xffffffffu,
                              mbar_wait_role(sm.odone(stream, half ^ 1), (half ? it : it - 1) & 1, fail));
              if (!ok) break;
              tcgen05_after_sync();
#pragma unroll 1
              for (int c = 0; c < 8; ++c) {
                float o[16];
                tmem_ld16(to + 16 * c, o);
                tmem_wait_ld16(o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] *= f;
                tmem_st16(to + 16 * c, reinterpret_cast<const uint32_t*>(o));
              }
            }
            sum *= f;
          }
          ref = next;
          careful = __any_sync(0xffffffffu, ref == -INFINITY || fabsf(ref) > kRefExact);
          const float rr = ref == -INFINITY ? 0.f : ref;
          const uint64_t r2 = f32x2(-rr, -rr);
#pragma unroll
          for (int e = 0; e < 64; e += 2) f32x2_split(add_f32x2(f32x2(v[e], v[e + 1]), r2), v[e], v[e + 1]);
          sum += pack_half(v, w);
          tmem_st32(ts + 32 * half, w);  // (over columns of S that both halves have left)
          arrive(half);
        }
      }
      if (!ok) break;
      ++it;
    }
    if (ok && it > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait_role(sm.odone(stream, 1), (it - 1) & 1, fail));
      tcgen05_after_sync();
    }
    float g0 = 1.f, g1 = 0.f;  // factors of this stream's and the other stream's O
    const float* other = reinterpret_cast<const float*>(smem_raw + (sm.stage(0) - smem_u32(smem_raw))) + r;
    // !PAIR: behind that O, the second stream's references, sums and marks
    float* other_ref = reinterpret_cast<float*>(smem_raw + (sm.stage(2) - smem_u32(smem_raw))) + r;
    if constexpr (!PAIR) {  // the second stream hands its part over through the (now unused) ring
      named_bar_sync(1, kSoftThreads);  // every MMA of both streams is done
      if (stream == 1) {
        other_ref[0] = it > 0 ? ref : -INFINITY;
        other_ref[kTile] = it > 0 ? sum : 0.f;
        other_ref[2 * kTile] = bad_row ? 1.f : 0.f;
        if (ok && it > 0) {
          float* to_first = const_cast<float*>(other);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float v[32];
            tmem_ld32(to + 32 * c, v);
            tmem_wait_ld(v);
#pragma unroll
            for (int e = 0; e < 32; ++e) to_first[(32 * c + e) * kTile] = v[e];
          }
        }
      }
      named_bar_sync(1, kSoftThreads);
      if (stream == 0) {
        const float r1 = other_ref[0], l1 = other_ref[kTile];
        bad_row = bad_row || other_ref[2 * kTile] != 0.f;
        const float top = fmaxf(ref, r1);
        if (top > -INFINITY) {
          g0 = fast_exp2(ref - top);
          g1 = fast_exp2(r1 - top);
        }
        sum = sum * g0 + l1 * g1;
        ref = top;
      }
    }
    if ((PAIR || stream == 0) && ok && !*fail) {
      const size_t out_row = ((size_t)b * a.tq + token) * a.heads_q + head;
      float lse2 = sum == 0.f ? -INFINITY : ref + log2f(sum);
      float f0 = sum == 0.f ? 0.f : 1.f / sum, f1 = 0.f;
      const bool last = p.n_splits == 1;
      if (last && a.own_out && valid) join_own(a, out_row, lse2, f0, f1);
      if (bad_row) f0 = __int_as_float(0x7fffffff);
      g0 *= f0;
      g1 *= f0;
      // (a row whose sum is 0 has seen nothing, or only scores of -inf: its O holds zeros or, never written, anything)
      const bool blank = f0 == 0.f;
      const bool other_ran = !PAIR && n_w[1] > 0;
      char* dst = last ? static_cast<char*>(a.out) +
                             (b * a.o_b + head * a.o_h + token * a.o_t) * (p.out_kind == 2 ? 4 : 2)
                       : reinterpret_cast<char*>(p.part_o + ((size_t)split * p.part_rows + out_row) * kHeadDim);
      const float* own = a.own_out + out_row * kHeadDim;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float v[32];
        if (it > 0) {
          tmem_ld32(to + 32 * c, v);
          tmem_wait_ld(v);
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          v[e] = blank ? 0.f : v[e] * g0;
          if (other_ran && !blank) v[e] = fmaf(other[(32 * c + e) * kTile], g1, v[e]);
        }
        if (valid) {
          if (f1 != 0.f) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 o = *reinterpret_cast<const float4*>(own + 32 * c + e);
              v[e] = fmaf(o.x, f1, v[e]);
              v[e + 1] = fmaf(o.y, f1, v[e + 1]);
              v[e + 2] = fmaf(o.z, f1, v[e + 2]);
              v[e + 3] = fmaf(o.w, f1, v[e + 3]);
            }
          }
#pragma unroll
          for (int e = 0; e < 32; e += 8) store_out8(dst, last ? p.out_kind : 2, 32 * c + e, v + e);
        }
      }
      if (valid) {
        if (last)
          store_stat(a, b * a.s_b + head * a.s_h + token * a.s_t, lse2);
        else
          p.part_lse[(size_t)split * p.part_rows + out_row] = lse2;
      }
    }
  }
  tcgen05_before_sync();
  __syncthreads();
  if (s_fail && tid == 0) record_error(a.status, kErrFullTimeout);
  if (warp == kMmaWarp) {
    __syncwarp();
    tcgen05_after_sync();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <bool F16, bool PAIR>
cudaError_t launch_variant(const FlashKernelArgs& p, dim3 grid, cudaStream_t st) {
  const bool cap = p.a.softcap > 0.f, bias = p.a.slopes != nullptr;
  auto k = cap ? (bias ? flash_kernel<F16, PAIR, true, true> : flash_kernel<F16, PAIR, true, false>)
               : (bias ? flash_kernel<F16, PAIR, false, true> : flash_kernel<F16, PAIR, false, false>);
  static std::atomic<uint64_t> configured[4];  // per variant: one bit per device
  std::atomic<uint64_t>& done = configured[2 * cap + bias];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev > 63 || !(done.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<PAIR>::kSmem);
    if (e != cudaSuccess) return e;
    done.fetch_or(bit, std::memory_order_relaxed);
  }
  k<<<grid, kThreads, Layout<PAIR>::kSmem, st>>>(p);
  return cudaGetLastError();
}

}  // namespace flash
}  // namespace mikv
