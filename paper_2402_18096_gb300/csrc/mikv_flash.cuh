// mikv_flash.cuh — attention over bf16 / fp16 keys on the fifth-generation tensor cores (sm_103a): the kernel
// template of the prompt and shared-prefix entry points. mikv_flash_bf16.cu and mikv_flash_f16.cu instantiate it for
// one operand type each; mikv_flash.cu holds the work plan, the merge of split parts and the dispatch.
//
// Problem. `batch` sets of keys; each set is attended by tq tokens of G query heads per KV head (a prompt's tokens are
// its positions, a shared prefix's tokens are its requests). The tq * G query rows of one KV head are packed into
// tiles of 128 rows, row R = token * G + head, so that all heads and tokens that share keys share their loads.
//
// Work. An item is a row tile (pair) of one KV head and set of keys. Where there are few of them, their key tiles are
// laid end to end and every CTA gets an equal run of them (a share): an item is then the part of a row tile's keys that
// lies in a CTA's share, and the parts are merged by a second kernel. A persistent CTA per SM takes items in turn, and
// its roles run ahead of one another across items: the next item's tiles are loaded and its first scores computed while
// the softmax warps still write the last item's output.
//
// A CTA has two streams, each with a score tile S (128 x 128 fp32) and an output tile O (128 x 128 fp32) in
// TMEM, over 128-key tiles of K and V that TMA stages in a ring:
//   kPair   two row tiles (256 rows) over the same key tiles: a K or V tile is loaded once for both.
//   kOne    one row tile (up to 128 rows) over alternating key tiles; the streams' results are joined at the end.
//           The second stream's loads and softmax overlap the first's, which keeps HBM busy when rows are few.
//   kFew    like kOne for up to 32 rows, which stand in the tile four times: each softmax warp then weighs a quarter
//           of a tile's keys for all rows (the others' weights are 0 in its copy), and the four copies of both streams
//           are joined at the end. One warp that weighs whole tiles takes longer than HBM takes to deliver them: with
//           capped and biased scores of 4 rows 5700 clocks for two tiles against 2700 a tile.
// Roles: warps 0-3 and 4-7 are the streams' softmax warpgroups (thread = row = TMEM lane), warp 8 issues the copies,
// warp 9 the MMAs, warp 10 guards masked tiles (below), warp 11 works out the coming items. Per stream and tile:
// S = Q K^T (8 MMAs of K = 16), softmax to P (16-bit, written over S in TMEM), O += P V (8 MMAs with A in TMEM). The MMA
// warp alternates streams, so one stream's softmax runs under the other's products. P lies over S and one warp
// issues all MMAs, which execute in the order of issue: the next tile's scores may be issued right behind the product
// that reads P. The MMA warp stays converged (elect_one) so that its operands stay in uniform registers: issuing from one
// lane's branch cost 80 clocks an MMA and a third of the rate.
//
// Barriers. Every role that waits on a barrier sees each of its phases in order (a wait that left phases out would
// take an earlier one of the same parity for its own); counters run on from item to item.
//
// Softmax. Weights are 2^(x - r) with x the score in log2 units and r a reference of the row: the largest x of 32 columns
// of its first tile, or of what it sees there where a mask cuts it (less ref_drop), moved only when a sum of weights
// passes sum_max, which rescales O. The
// weights' 16-bit types hold that range without loss of relative precision, so most tiles need no maximum at all. Key
// tiles are visited from the last to the first: with a causal mask or a distance bias the largest scores then
// tend to come first. Sums are fp32 over the unrounded weights; rounding the weights to 16 bits is what the tensor
// cores take, and perturbs each weight by at most half a unit in its last place.
//
// Masks. Every row sees one span of keys [lo, hi). Tiles outside the union of an item's spans are not visited; tiles
// inside every span are not masked. In the tiles between, a weight of 0 does not stop an infinity or NaN in V from
// entering O (0 * inf), so the guard warp looks through the V tile first: rows with such a value are set to 0 and
// their keys reported to the softmax threads, which mark the output rows that do see them. In tiles that no mask cuts an
// infinity reaches the rows as the products give it: infinite, or NaN where its weight rounds to 0 (as in kFew, whose
// copies weigh three quarters of the keys by 0).
//
// Bounds. Two row tiles take at least 2068 clocks of the tensor cores per key tile (4 x 128^3 at 517 each, measured alone)
// and about 2900 in the kernel: what is left is the chain of one stream (scores -> softmax, about 1200 clocks -> product
// and next scores, 1034, and two hand-overs), which two streams in 512 TMEM columns cannot hide altogether. Causal, T 8192,
// 32 query and 8 KV heads: 345 us, 1.59 PFLOP/s. A cap adds an exponential and a quarter of a reciprocal per score
// (1.00 PFLOP/s at the same size), a distance bias an addition (1.47). With one row tile a set's keys pass once:
// HBM. 8 requests of 32 heads with 4096 keys of their own: 86 us, 6.3 TB/s (92 % of a copy).
//
// Code that runs once per item or launch is bound by fetching its instructions (traces: 2 us from the start of a CTA to its
// first item, 2.5 us for the output of one), so such code is kept in loops, and each path has one form: a kernel of 131 KB
// of code took 88 us where its 88 KB form took 84 (four prompts of other lengths, 16 requests, cap and bias).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <limits.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "mikv_device.cuh"
#include "mikv_flash.h"
#include "mikv_internal.h"
#include "mikv_tcgen05.cuh"

namespace mikv {

template <bool F16>
cudaError_t launch_flash_kernel(const FlashKernelArgs& p, int mode, int grid, cudaStream_t st);

namespace flash {

constexpr int kTile = 128;                     // query rows of a tile, keys of a tile
constexpr int kTileBytes = kTile * kHeadDim * 2;
constexpr int kHalfBytes = kTileBytes / 2;     // one 64-channel box
constexpr int kSoftThreads = 256;
constexpr int kCopyWarp = 8, kMmaWarp = 9, kGuardWarp = 10;  // 11: the items'
constexpr int kExPitch = 68;                   // floats of a row's 64 channels in the exchange (padded against conflicts)
constexpr int kItemRing = 4;                   // items described ahead
constexpr int kItemReaders = 11;               // warps that read an item's description: all but the one that writes it
constexpr int kThreads = 384;
constexpr int kTmemCols = 512;                 // S0, S1, O0, O1
constexpr int kSafeRing = 4;                   // guard results in flight (more than V tiles of a stream in the ring)
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__host__ __device__ constexpr int align16(int x) { return (x + 15) & ~15; }

enum Mode { kPair = 0, kOne = 1, kFew = 2 };

template <int MODE>
struct Layout {
  static constexpr bool PAIR = MODE == kPair;
  static constexpr int kCopies = MODE == kFew ? 4 : 1;   // of the rows in a tile
  static constexpr int kRows = kTile / kCopies;          // rows of a tile
  static constexpr int kItemRows = (PAIR ? 2 : 1) * kRows;  // rows of an item
  static constexpr int kExchange = MODE == kFew ? 8 * 8 * kExPitch * 4 : 0;  // for joining the copies
  static constexpr int kQ = PAIR ? 2 : 1;  // query tiles in shared memory
  static constexpr int kStages = 5;        // K / V tiles in the ring
  // Loads of an item: the first kLead K tiles, then V tile u and K tile u + kLead for u = 0, 1, ... (from the last
  // key tile on).
  static constexpr int kLead = PAIR ? 1 : 2;
  static constexpr int kBars = 2 + 2 * kStages + 5 * 2 + 2 * kSafeRing + 2 * kItemRing + 1;
  static constexpr int kSmem = 1024 + (kQ + kStages) * kTileBytes + align16(8 * kBars) + kExchange;
  static_assert(kSmem <= 224 * 1024 + 2048, "shared memory of one CTA");
  uint32_t base;
  __device__ uint32_t q(int m) const { return base + m * kTileBytes; }
  __device__ uint32_t stage(int s) const { return base + (kQ + s) * kTileBytes; }
  __device__ uint32_t bar(int i) const { return base + (kQ + kStages) * kTileBytes + 8 * i; }
  __device__ uint32_t exchange() const { return base + (kQ + kStages) * kTileBytes + align16(8 * kBars); }
  __device__ uint32_t qfull() const { return bar(0); }                       // an item's queries landed
  __device__ uint32_t qfree() const { return bar(1); }                       // its last scores have read them
  __device__ uint32_t full(int s) const { return bar(2 + s); }               // a copy landed
  __device__ uint32_t empty(int s) const { return bar(2 + kStages + s); }    // it is not needed any more
  __device__ uint32_t sfull(int w) const { return bar(2 + 2 * kStages + w); }  // scores of stream w
  // of half a tile (64 keys): weights written (and O rescaled for them); O += P V done
  __device__ uint32_t pready(int w, int half) const { return bar(4 + 2 * kStages + 2 * w + half); }
  __device__ uint32_t odone(int w, int half) const { return bar(8 + 2 * kStages + 2 * w + half); }
  // guarded V tile looked through (PAIR: set 0 serves both streams)
  __device__ uint32_t vsafe(int w, int g) const { return bar(12 + 2 * kStages + kSafeRing * w + g % kSafeRing); }
  // an item's description written; read by every role
  __device__ uint32_t itemfull(int i) const { return bar(12 + 2 * kStages + 2 * kSafeRing + i % kItemRing); }
  __device__ uint32_t itemfree(int i) const { return bar(12 + 2 * kStages + 2 * kSafeRing + kItemRing + i % kItemRing); }
  __device__ uint32_t drain() const { return bar(kBars - 1); }
  // Arrivals that complete a phase of barrier i.
  __device__ static constexpr int arrivals(int i) {
    if (i >= 2 + kStages && i < 2 + 2 * kStages) return 2;           // empty: its MMAs and the guard warp
    if (i >= 4 + 2 * kStages && i < 8 + 2 * kStages) return 4;       // pready: the softmax warps of the stream
    if (i >= 12 + 2 * kStages + 2 * kSafeRing + kItemRing && i < kBars - 1) return kItemReaders;  // itemfree
    return 1;
  }
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
  int pos;           // its position
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

// The cap of four scores: cap tanh(y) + rest = cap (e - 1) / (e + 1) + rest with e = e^2y. One reciprocal serves all
// four: with p = (ac, bd) of the denominators a, b, c, d, 1 / a = bd c / (ac bd) and so on. 2^30 stands for larger
// exponentials (tanh is then 1 to fp32 precision), which keeps the product of four inside fp32. For small y, e - 1 is
// exact and the quotient's roundings are relative to it: only the exponential's own error, 2^-23 of cap, remains.
__device__ __forceinline__ void cap_four(float* v, float scale, float cap, uint64_t rest0, uint64_t rest1) {
  const uint64_t s2 = f32x2(scale, scale), one = f32x2(1.f, 1.f), less = f32x2(-1.f, -1.f), c2 = f32x2(cap, cap);
  float y[4];
  f32x2_split(mul_f32x2(f32x2(v[0], v[1]), s2), y[0], y[1]);
  f32x2_split(mul_f32x2(f32x2(v[2], v[3]), s2), y[2], y[3]);
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = fast_exp2(min_nan(y[i], 30.f));
  const uint64_t e0 = f32x2(y[0], y[1]), e1 = f32x2(y[2], y[3]);
  const uint64_t ab = add_f32x2(e0, one), cd = add_f32x2(e1, one);
  float ac, bd;
  f32x2_split(mul_f32x2(ab, cd), ac, bd);
  const float r = rcp_approx(ac * bd);
  const uint64_t s = mul_f32x2(f32x2(r, r), f32x2(bd, ac));
  const uint64_t t0 = mul_f32x2(mul_f32x2(s, cd), add_f32x2(e0, less));
  const uint64_t t1 = mul_f32x2(mul_f32x2(s, ab), add_f32x2(e1, less));
  f32x2_split(fma_f32x2(t0, c2, rest0), v[0], v[1]);
  f32x2_split(fma_f32x2(t1, c2, rest1), v[2], v[3]);
}

__device__ __forceinline__ float max3(float a, float b, float c) {  // NaN operands are passed over
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// N scores (columns col0 .. of the tile at key k0) less `ref`, in place.
// LINEAR: all the keys lie on one side of the row's position, and the bias is slope times (key - position).
template <bool CAP, bool BIAS, int N, bool LINEAR>
__device__ __forceinline__ void row_scores(float* v, const Score& sc, const Row& row, int k0, int col0, float ref,
                                           float slope) {
  const float rest = -ref;
  auto apply = [&](auto bias) {  // bias(i): the biases of columns i and i + 1, plus `rest`
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint64_t b0 = bias(i), b1 = bias(i + 2);
      if constexpr (CAP) {
        cap_four(v + i, sc.scale, sc.cap, b0, b1);
      } else {
        const uint64_t s2 = f32x2(sc.scale, sc.scale);
        f32x2_split(fma_f32x2(f32x2(v[i], v[i + 1]), s2, b0), v[i], v[i + 1]);
        f32x2_split(fma_f32x2(f32x2(v[i + 2], v[i + 3]), s2, b1), v[i + 2], v[i + 3]);
      }
    }
  };
  if constexpr (!BIAS) {
    apply([&](int) { return f32x2(rest, rest); });
  } else {
    const float e0 = (float)(int)((unsigned)(k0 + col0) - (unsigned)row.pos);  // (exact up to distances of 2^24)
    if constexpr (LINEAR) {
      uint64_t near[4];  // within eight columns, which share a base
#pragma unroll
      for (int k = 0; k < 4; ++k) near[k] = f32x2(slope * (2.f * k), slope * (2.f * k + 1.f));
      apply([&](int i) {
        const float base = fmaf(slope, e0 + (float)(i & ~7), rest);
        return add_f32x2(f32x2(base, base), near[(i & 7) / 2]);
      });
    } else {
      apply([&](int i) {
        return f32x2(fmaf(-slope, fabsf(e0 + (float)i), rest), fmaf(-slope, fabsf(e0 + (float)(i + 1)), rest));
      });
    }
  }
}

// The keys of [first_key, first_key + 32) that the row sees, a bit each.
__device__ __forceinline__ uint32_t seen_keys(const Row& row, int first_key) {
  const int end = min(max(row.hi - first_key, 0), 32), first = min(max(row.lo - first_key, 0), 32);
  return (uint32_t)((1ull << end) - 1) & ~(uint32_t)((1ull << first) - 1);
}
// 32 scores, replaced by x where the row does not see the key (a test of a bit and a move each).
__device__ __forceinline__ void mask_scores(float* v, uint32_t seen, float x) {
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (!(seen & (1u << i))) v[i] = x;
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

// 32 outputs at element i of an output row, in stores of a whole 32-byte sector where the row is aligned for it.
__device__ __forceinline__ void store32(void* at, const uint32_t (&v)[8], bool aligned32) {
  if (aligned32) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                 "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
    static_cast<uint4*>(at)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    static_cast<uint4*>(at)[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
}
template <bool F16>
__device__ __forceinline__ void store_out32(char* row, bool f32, int i, const float (&v)[32]) {
  const bool al = (reinterpret_cast<uintptr_t>(row) & 31) == 0;
  uint32_t u[8];
  if (f32) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = __float_as_uint(v[8 * q + e]);
      store32(row + 4 * (i + 8 * q), u, al);
    }
  } else {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        u[e] = pack16<F16>(v[16 * q + 2 * e], v[16 * q + 2 * e + 1]);
      store32(row + 2 * (i + 16 * q), u, al);
    }
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

// One item of work: its place, per stream the key tiles [t0, t1) that some row sees and the keys that every row sees, and
// this item's share [T0, T1) of the union of both streams' tiles. As it lies in shared memory.
struct alignas(16) ItemData {
  int b, h, m_block, slot;  // slot: where the part of a share goes
  int t0[2], t1[2];
  int all_lo[2], all_hi[2];
  int T0, T1;
  int valid, unused;
};

template <bool PAIR>
struct Item : ItemData {
  int n;
  __device__ static int of(const int (&x)[2], int w) { return w ? x[1] : x[0]; }
  __device__ bool active(int w, int j) const { return !PAIR || (j >= of(t0, w) && j < of(t1, w)); }
  __device__ bool cut(int w, int j) const { return j * kTile < of(all_lo, w) || (j + 1) * kTile > of(all_hi, w); }
  __device__ bool guarded(int j) const {
    return PAIR ? (active(0, j) && cut(0, j)) || (active(1, j) && cut(1, j)) : cut(0, j);
  }
  __device__ int tiles_of(int w) const { return PAIR ? n : w ? n / 2 : (n + 1) / 2; }  // visited by stream w
};

// Place of item number `index` among whole row tiles. Heads go in groups whose keys fit in L2 together; within a group a
// causal prompt's longest rows come first.
__device__ __forceinline__ ItemData place_at(const FlashKernelArgs& p, int index) {
  const FlashArgs& a = p.a;
  ItemData x = {};
  const int group = p.by_group.div(index);
  int rest = index - group * p.by_group.d;
  const bool last = (group + 1) * p.group_heads > a.batch * a.heads_kv;  // (a smaller group)
  const int rank = last ? p.by_last.div(rest) : p.by_rank.div(rest);
  rest -= rank * (last ? p.by_last.d : p.by_rank.d);
  const int bh = group * p.group_heads + rest;
  x.b = p.by_head.div(bh);
  x.h = bh - x.b * a.heads_kv;
  x.m_block = p.m_blocks - 1 - rank;
  return x;
}

// The key tiles of an item whose place is known, worked out by a whole warp (the same in every lane).
template <int MODE>
__device__ __forceinline__ void item_tiles(const FlashKernelArgs& p, ItemData& x, int lane) {
  constexpr bool PAIR = MODE == kPair;
  const FlashArgs& a = p.a;
  x.valid = 1;
  const int toks = Layout<MODE>::kRows / a.G;
  constexpr int W = PAIR ? 2 : 1;
  // what the tokens of each tile see: their union [lo, hi) (hi = 0: none), and what all of them see
  int lo[W], hi[W], all_lo[W], all_hi[W];
  if (a.spans) {
    int2 s[W][4];  // up to 128 tokens of a tile, four to a lane; all loads in flight
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = lane + 32 * i, t = (PAIR ? 2 * x.m_block + w : x.m_block) * toks + at;
        if (at < toks && t < a.tq) s[w][i] = __ldg(a.spans + (size_t)x.b * a.tq + t);
      }
#pragma unroll
    for (int w = 0; w < W; ++w) {
      lo[w] = INT_MAX, hi[w] = 0, all_lo[w] = 0, all_hi[w] = INT_MAX;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = lane + 32 * i;
        if (at >= toks || (PAIR ? 2 * x.m_block + w : x.m_block) * toks + at >= a.tq) continue;
        const int l = max(s[w][i].x, 0), h = min(s[w][i].y, a.tk);
        const bool sees = h > l;
        lo[w] = min(lo[w], sees ? l : INT_MAX);
        hi[w] = max(hi[w], sees ? h : 0);
        all_lo[w] = max(all_lo[w], sees ? l : INT_MAX);
        all_hi[w] = min(all_hi[w], sees ? h : 0);
      }
      lo[w] = __reduce_min_sync(0xffffffffu, lo[w]);
      hi[w] = __reduce_max_sync(0xffffffffu, hi[w]);
      all_lo[w] = __reduce_max_sync(0xffffffffu, all_lo[w]);
      all_hi[w] = __reduce_min_sync(0xffffffffu, all_hi[w]);
    }
  } else {
    const int len = a.lens ? max(0, min(a.lens[x.b], a.tk)) : a.tk;
#pragma unroll
    for (int w = 0; w < W; ++w) {  // every token sees [0, its end), and the ends do not fall
      const int tok0 = (PAIR ? 2 * x.m_block + w : x.m_block) * toks, tok1 = min(tok0 + toks, a.tq);
      int first = len, end = len;
      if (a.causal) {
        first = (int)min((long long)len, max(0ll, (long long)a.q_start + tok0 + 1));
        end = (int)min((long long)len, max(0ll, (long long)a.q_start + tok1));
      }
      const bool any = tok0 < tok1;
      lo[w] = any && end > 0 ? 0 : INT_MAX;
      hi[w] = any ? end : 0;
      all_lo[w] = any && first == 0 ? INT_MAX : 0;
      all_hi[w] = any ? first : INT_MAX;
    }
  }
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int v = w < W ? w : 0;
    x.t0[w] = hi[v] > 0 ? lo[v] / kTile : INT_MAX;
    x.t1[w] = (hi[v] + kTile - 1) / kTile;
    x.all_lo[w] = all_lo[v];
    x.all_hi[w] = all_hi[v];
  }
  x.T0 = min(x.t0[0], x.t0[1]);
  x.T1 = max(x.t1[0], x.t1[1]);
  if (x.T1 == 0) x.T0 = 0;
}

// Units (key tiles) are numbered set by set, head by head, row block by row block; CTA c has the units [first(c),
// first(c + 1)), one more for the first `extra` CTAs.
struct Shares {
  int each, extra;
  __device__ int first(int c) const { return c * each + min(c, extra); }
  __device__ int owner(int u) const {
    const int big = extra * (each + 1);
    return u < big ? u / (each + 1) : extra + (u - big) / each;
  }
};
// Units of every row block of set b: its key tiles where they follow from the set's length, else those of all keys (and a
// part takes the same fraction of the tiles that the row block really has).
__device__ __forceinline__ int units_of(const FlashKernelArgs& p, int b) {
  return p.by_length ? (max(0, min(p.a.lens[b], p.a.tk)) + kTile - 1) / kTile : p.units;
}

// Items of this CTA: one of every gridDim.x, alternately from the front and from the back of a round, which evens out
// the lengths of a causal prompt's rows.
__device__ __forceinline__ int item_index(int round) {
  return round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

// Barrier of the softmax warps that tells all of them whether one of them (or another role) has failed.
__device__ __forceinline__ bool softmax_sync(bool failed) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)failed), "n"(kSoftThreads)
      : "memory");
  return any != 0;
}

template <bool F16, int MODE, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) flash_kernel(const __grid_constant__ FlashKernelArgs p) {
  using L = Layout<MODE>;
  constexpr bool PAIR = L::PAIR;
  const FlashArgs& a = p.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;
  __shared__ ItemData s_item[kItemRing];
  __shared__ uint32_t s_bad[2][kSafeRing][4];  // keys of a guarded V tile that hold infinities or NaN
  // !PAIR: reference and sum of each part of a row, and whether it saw an infinity or NaN. Part: stream and copy.
  __shared__ float s_part[2 * L::kCopies][2][L::kRows];
  __shared__ uint8_t s_mark[2 * L::kCopies][L::kRows];
  volatile int* fail = &s_fail;
  L sm;
  sm.base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

  if (tid < L::kBars) mbar_init(sm.bar(tid), L::arrivals(tid));
  if (tid == 0) s_fail = 0;
  fence_mbar_init();
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&s_tmem), kTmemCols);
  if (tid == 32 * kCopyWarp) {
    prefetch_tensormap(&p.map_q);
    prefetch_tensormap(&p.map_k);
    prefetch_tensormap(&p.map_v);
  }
  tcgen05_before_sync();
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
  grid_dependency_wait();
  if (p.shares) allow_dependent_launch();  // (the merge; CTAs of the next grid that wait on freed SMs slow the rest of whole tiles)
  // The description of the item of a round (uniform); false when a wait gave up.
  auto next_item = [&](int round, Item<PAIR>& x) {
    const bool ok = mbar_wait_warp(sm.itemfull(round), (round / kItemRing) & 1, fail);
    const int* d = reinterpret_cast<const int*>(&s_item[round % kItemRing]);
    int* to = reinterpret_cast<int*>(static_cast<ItemData*>(&x));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(ItemData) / 4); ++i) to[i] = __shfl_sync(0xffffffffu, d[i], 0);
    x.n = x.T1 - x.T0;
    __syncwarp();
    if (lane == 0) mbar_arrive(sm.itemfree(round));
    return ok;
  };

  // The softmax warps take the registers the other warpgroup does not need: 256 x 216 + 128 x 72 = 384 x 168.
  if (warp >= kCopyWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    int c = 0;        // loads so far
    int running = 0;  // items with key tiles so far
    if (warp == kCopyWarp) {
      int last[L::kStages];  // the last load of each stage
#pragma unroll
      for (int s = 0; s < L::kStages; ++s) last[s] = -1;
      bool ok = true;
      Item<PAIR> x;
      for (int round = 0; ok; ++round) {
        ok = next_item(round, x);
        if (!ok || !x.valid) break;
        if (x.n == 0) continue;
        if (lane == 0) {
          auto load_q = [&]() {
            if (running > 0 && !mbar_wait_role(sm.qfree(), (running - 1) & 1, fail)) return false;
            mbar_arrive_expect_tx(sm.qfull(), L::kQ * kTileBytes);
#pragma unroll
            for (int m = 0; m < L::kQ; ++m) {
              const int tok0 = (PAIR ? 2 * x.m_block + m : x.m_block) * (kTile / a.G);
#pragma unroll 1
              for (int copy = 0; copy < L::kCopies; ++copy) {
                const uint32_t to = sm.q(m) + copy * L::kRows * 128;
                tma_load_4d(to, &p.map_q, 0, x.h * a.G, tok0, x.b, sm.qfull());
                tma_load_4d(to + kHalfBytes, &p.map_q, 64, x.h * a.G, tok0, x.b, sm.qfull());
              }
            }
            ++running;
            return true;
          };
          // V tile u, then K tile u + kLead; the first kLead K tiles and the queries before them
#pragma unroll 1
          for (int i = -2 * L::kLead; ok && i < 2 * x.n; ++i) {
            const int u = i >> 1;
            const bool keys = i & 1;
            if (i == 0) ok = load_q();
            if (keys ? u + L::kLead >= x.n : u < 0) continue;
            const int s = c % L::kStages, j = (x.T1 - 1 - u - (keys ? L::kLead : 0)) * kTile;
            const CUtensorMap* map = keys ? &p.map_k : &p.map_v;
            const int h = x.h * (keys ? p.k_head : p.v_head), b = x.b * (keys ? p.k_batch : p.v_batch);
            ok = ok && (c < L::kStages || mbar_wait_role(sm.empty(s), ((c / L::kStages) & 1) ^ 1, fail));
            if (!ok) break;
            mbar_arrive_expect_tx(sm.full(s), kTileBytes);
            tma_load_4d(sm.stage(s), map, 0, j, h, b, sm.full(s));
            tma_load_4d(sm.stage(s) + kHalfBytes, map, 64, j, h, b, sm.full(s));
#pragma unroll
            for (int q = 0; q < L::kStages; ++q)
              if (q == s) last[q] = c;
            ++c;
          }
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
      }
      if (lane == 0) {  // no copy may outlive the CTA, whatever became of the other roles
        if (running > 0 && !mbar_wait(sm.qfull(), (running - 1) & 1)) record_error(a.status, kErrDrainTimeout);
#pragma unroll
        for (int s = 0; s < L::kStages; ++s)
          if (last[s] >= 0 && !mbar_wait(sm.full(s), (last[s] / L::kStages) & 1)) record_error(a.status, kErrDrainTimeout);
      }
      __syncwarp();
    } else if (warp == kMmaWarp) {  // the whole warp, converged; one lane issues
      const bool leader = elect_one();
      int tiles[2] = {0, 0};    // tiles of each stream whose weights were consumed
      int checked[2] = {0, 0};  // guarded tiles (PAIR: in checked[0])
      auto of = [](const int(&x)[2], int w) { return w ? x[1] : x[0]; };
      auto commit = [&](uint32_t bar) {
        if (leader) umma_commit(bar);
      };
      auto wait_full = [&](int load) {
        const bool ok = mbar_wait_warp(sm.full(load % L::kStages), (load / L::kStages) & 1, fail);
        tcgen05_after_sync();
        return ok;
      };
      auto release = [&](int load) { commit(sm.empty(load % L::kStages)); };
      auto scores = [&](int w, int load) {
        const uint32_t q = sm.q(PAIR ? w : 0), k = sm.stage(load % L::kStages);
        if (leader) {
          mma_scores<F16>(tmem + 128 * w, q, k);
          umma_commit(sm.sfull(w));
        }
      };
      auto values = [&](int w, int load, bool first) {
        const uint32_t v = sm.stage(load % L::kStages);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!mbar_wait_warp(sm.pready(w, half), of(tiles, w) & 1, fail)) return false;
          tcgen05_after_sync();
          if (leader) {
            mma_values<F16>(tmem + 256 + 128 * w, tmem + 128 * w, v, half, !first);
            umma_commit(sm.odone(w, half));
          }
        }
        (w ? tiles[1] : tiles[0]) += 1;
        return true;
      };
      auto wait_safe = [&](int w) {
        const int g = of(checked, w);
        (w ? checked[1] : checked[0]) += 1;
        return mbar_wait_warp(sm.vsafe(w, g), (g / kSafeRing) & 1, fail);
      };
      bool ok = true;
      Item<PAIR> x;
      for (int round = 0; ok; ++round) {
        ok = next_item(round, x);
        if (!ok || !x.valid) break;
        const int n = x.n;
        if (n == 0) continue;
        ok = mbar_wait_warp(sm.qfull(), running & 1, fail);
        ++running;
        if constexpr (PAIR) {
          bool fresh[2] = {true, true};  // the stream's O holds nothing of this item yet
          ok = ok && wait_full(c);
          if (ok) {
#pragma unroll
            for (int w = 0; w < 2; ++w)
              if (x.active(w, x.T1 - 1)) scores(w, c);
            release(c);
            if (n == 1) commit(sm.qfree());
          }
          for (int i = 0; ok && i < n; ++i) {
            const int j = x.T1 - 1 - i, cv = c + 1, ck = c + 2;
            ok = wait_full(cv) && (!x.guarded(j) || wait_safe(0));
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              if (ok && x.active(w, j)) {
                ok = values(w, cv, fresh[w]);
                fresh[w] = false;
              }
              if (ok && i + 1 < n) {
                if (w == 0) ok = wait_full(ck);
                if (ok && x.active(w, j - 1)) scores(w, ck);
              }
            }
            if (ok) {
              release(cv);
              if (i + 1 < n) release(ck);
              if (i + 2 == n) commit(sm.qfree());
            }
            c += 2;
          }
        } else {  // step u: the product of tile u (from 0 on), then the scores of tile u + 2; streams in turn
#pragma unroll 1
          for (int u = -2; ok && u < n; ++u) {
            const int w = u & 1;
            if (u >= 0) {
              ok = wait_full(c) && (!x.guarded(x.T1 - 1 - u) || wait_safe(w)) && values(w, c, u < 2);
              if (ok) {
                release(c);
                ++c;
              }
            }
            if (ok && u + 2 < n) {
              ok = wait_full(c);
              if (ok) {
                scores(w, c);
                release(c);
                ++c;
                if (u + 3 == n) commit(sm.qfree());
              }
            }
          }
        }
      }
      commit(sm.drain());  // every MMA issued has completed once this arrives
      if (!mbar_wait(sm.drain(), 0) && lane == 0) record_error(a.status, kErrDrainTimeout);
      __syncwarp();
    } else if (warp == kGuardWarp) {  // it sees every load in order, looks through guarded V tiles, releases each load too
      int checked[2] = {0, 0};
      auto of = [](const int(&x)[2], int w) { return w ? x[1] : x[0]; };
      auto landed = [&]() { return mbar_wait_warp(sm.full(c % L::kStages), (c / L::kStages) & 1, fail); };
      auto release = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.empty(c % L::kStages));
        ++c;
      };
      bool ok = true;
      Item<PAIR> x;
      for (int round = 0; ok; ++round) {
        ok = next_item(round, x);
        if (!ok || !x.valid) break;
        const int n = x.n;
        for (int u = 0; ok && u < min(n, L::kLead); ++u) {
          ok = landed();
          if (ok) release();
        }
        for (int u = 0; ok && u < n; ++u) {
          const int j = x.T1 - 1 - u, w = PAIR ? 0 : u & 1;
          ok = landed();
          if (!ok) break;
          if (x.guarded(j)) {
            const int g = of(checked, w);
            bool wrote = false;
#pragma unroll 1
            for (int part = 0; part < 4; ++part) {
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
    } else {  // the coming items, up to kItemRing ahead, and the end (little code: every launch fetches it anew)
      int round = 0;
      auto publish = [&](const ItemData& x) {
        if (round >= kItemRing && !mbar_wait_warp(sm.itemfree(round), ((round / kItemRing) & 1) ^ 1, fail)) return false;
        if (lane == 0) {
          s_item[round % kItemRing] = x;
          mbar_arrive(sm.itemfull(round));
        }
        __syncwarp();
        ++round;
        return true;
      };
      // Shares: this CTA's units [lo, hi); the row block that holds the next unit `u`: set b, number `in_set` in it, first
      // unit `start`.
      const int per_set = a.heads_kv * p.m_blocks;
      Shares sh = {p.share_each, p.share_extra};
      int b = 0, in_set = 0, start = 0, u = 0, hi = 0;
      if (p.shares && !p.by_length) {
        u = sh.first(blockIdx.x), hi = sh.first(blockIdx.x + 1);
        const int m = p.by_units.div(u);
        b = p.by_set.div(m);
        in_set = m - b * per_set;
        start = m * p.units;
      } else if (p.shares) {
        auto scan = [&](int b0, int& mine) {  // units of the sets b0 .. b0 + lane, and of this lane's
          mine = b0 + lane < a.batch ? units_of(p, b0 + lane) * per_set : 0;
          int sum = mine;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += y;
          }
          return sum;
        };
        int all = 0, mine, sum;
#pragma unroll 1
        for (int b0 = 0; b0 < a.batch; b0 += 32) all += __shfl_sync(0xffffffffu, scan(b0, mine), 31);
        sh.each = all / (int)gridDim.x;
        sh.extra = all - sh.each * gridDim.x;
        u = sh.first(blockIdx.x), hi = sh.first(blockIdx.x + 1);
        int before = 0;
#pragma unroll 1
        for (int b0 = 0; u < hi && b0 < a.batch; b0 += 32) {
          sum = scan(b0, mine);
          const int total = __shfl_sync(0xffffffffu, sum, 31);
          if (u < before + total) {
            const int at = __ffs(__ballot_sync(0xffffffffu, before + sum > u)) - 1;
            b = b0 + at;
            start = before + __shfl_sync(0xffffffffu, sum - mine, at);
            const int t = units_of(p, b);
            in_set = (u - start) / t;
            start += in_set * t;
            break;
          }
          before += total;
        }
      }
      bool ok = true;
#pragma unroll 1
      while (ok) {
        ItemData x = {};
        int t = 0;  // units of the row block
        if (!p.shares) {
          const int index = item_index(round);
          if (index >= p.n_items) break;
          x = place_at(p, index);
        } else {
          if (u >= hi) break;
          t = units_of(p, b);
          x.b = b;
          x.h = p.by_block.div(in_set);
          x.m_block = in_set - x.h * p.m_blocks;
          x.slot = blockIdx.x + b * per_set + in_set;
        }
        item_tiles<MODE>(p, x, lane);
        if (p.shares) {
          const int from = u - start, end = min(hi - start, t);
          if (!p.by_length) {  // units to tiles: a rising function, the same for the part before and the one behind
            const int n = x.T1 - x.T0;
            auto tile = [&](int unit) { return unit == t ? n : min(n, (int)((float)n * (float)unit * p.inv_units)); };
            x.T1 = x.T0 + tile(end);
            x.T0 += tile(from);
          } else {
            x.T1 = x.T0 + end;
            x.T0 += from;
          }
          u = start + end;
          if (end == t) {  // on to the next row block that has units
            start += t;
            if (++in_set == per_set) {
              in_set = 0;
              do ++b;
              while (b < a.batch && units_of(p, b) == 0);
            }
          }
        }
        ok = publish(x);
      }
      if (ok) publish(ItemData{});
      if (p.shares && blockIdx.x == 0) {  // for the merge: the first CTA of each row block, and how many share it
        int unit = 0;
#pragma unroll 1
        for (int set = 0; set < a.batch; ++set) {
          const int t = units_of(p, set);
#pragma unroll 1
          for (int i = lane; i < per_set; i += 32) {
            const int u0 = unit + i * t, first = t > 0 ? sh.owner(u0) : 0;
            p.part_table[set * per_set + i] = make_int2(first, t > 0 ? sh.owner(u0 + t - 1) - first + 1 : 0);
          }
          unit += per_set * t;
        }
      }
    }
  } else {  // softmax warps
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int stream = warp >> 2, r = tid & (L::kRows - 1);
    const int part = MODE == kFew ? warp : stream;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t ts = tmem + 128 * stream + lanes, to = tmem + 256 + 128 * stream + lanes;
    Score sc;
    sc.scale = CAP ? 2.f * kLog2e * (a.sm_scale / a.softcap) : a.sm_scale * kLog2e;
    sc.cap = a.softcap * kLog2e;
    int tiles = 0, guards = 0;  // tiles done and guarded tiles met, over all items
    Item<PAIR> x;
    // What the thread's row of an item needs from memory, asked for ahead of its use.
    int token = 0, head = 0;
    int2 span = make_int2(0, 0);
    int length = 0, at = 0;
    float slope = 0.f;
    auto load_row = [&]() {
      const int R = (PAIR ? 2 * x.m_block + stream : x.m_block) * L::kRows + r;
      token = R >> p.log2_G;
      head = x.h * a.G + (R & (a.G - 1));
      if (token >= a.tq) return;
      if (a.lens) length = a.lens[x.b];
      if (a.spans) span = a.spans[(size_t)x.b * a.tq + token];
      if constexpr (BIAS) {
        if (a.pos) at = a.pos[(size_t)x.b * a.tq + token];
        slope = a.slopes[head];
      }
    };
    bool ok = next_item(0, x);
    if (ok && x.valid) load_row();
    if (!PAIR) ok = !softmax_sync(!ok);  // (all of them go on, or none)
    for (int round = 0; ok && x.valid; ++round) {
      const bool valid = token < a.tq;
      Row row;
      row.lo = row.hi = 0;
      row.pos = 0;
      row.slope = 0.f;
      int pos = 0;
      if (valid) {
        const int len = a.lens ? max(0, min(length, a.tk)) : a.tk;
        row.hi = len;
        if (a.spans) {
          row.lo = max(span.x, 0);
          row.hi = min(span.y, a.tk);
        } else if (a.causal) {
          row.hi = (int)min((long long)len, max(0ll, (long long)a.q_start + token + 1));
        }
        if constexpr (BIAS) {
          pos = a.pos ? at : a.pos_at_len ? len : a.q_start + token;
          row.pos = pos;
          row.slope = slope * kLog2e;
        }
        if (row.hi <= row.lo) row.lo = row.hi = 0;
      }
      const bool sees = row.hi > row.lo;
      const int warp_lo = __reduce_min_sync(0xffffffffu, sees ? row.lo : INT_MAX);
      const int warp_hi = __reduce_max_sync(0xffffffffu, row.hi);
      const int warp_all_lo = __reduce_max_sync(0xffffffffu, !valid ? 0 : sees ? row.lo : INT_MAX);
      const int warp_all_hi = __reduce_min_sync(0xffffffffu, !valid ? INT_MAX : row.hi);
      int pos_min = 0, pos_max = 0;
      if (BIAS) {
        pos_min = __reduce_min_sync(0xffffffffu, valid ? pos : INT_MAX);
        pos_max = __reduce_max_sync(0xffffffffu, valid ? pos : INT_MIN);
      }
      const bool any_valid = __any_sync(0xffffffffu, valid);
      // (a row that sees nothing, or past the last token, needs no reference: its weights are 0 or never used)
      float ref = sees ? -INFINITY : 0.f, sum = 0.f;
      bool bad_row = false;
      bool careful = true;  // some row of the warp has no reference yet, or one beyond kRefExact
      int it = 0;           // tiles of this item done
      for (int i = 0; i < x.tiles_of(stream); ++i) {
        const int j = x.T1 - 1 - (PAIR ? i : 2 * i + stream);
        const bool guarded = x.guarded(j);
        if (guarded) ++guards;
        if (!x.active(stream, j)) continue;
        const int k0 = j * kTile;
        ok = __all_sync(0xffffffffu, mbar_wait_role(sm.sfull(stream), tiles & 1, fail));
        if (!ok) break;
        tcgen05_after_sync();
        auto arrive = [&](int first, int n) {
          tmem_wait_st();
          tcgen05_before_sync();
          __syncwarp();
          if (lane == 0)
            for (int half = first; half < first + n; ++half) mbar_arrive(sm.pready(stream, half));
        };
        if (k0 >= warp_hi || k0 + kTile <= warp_lo) {  // no row of this warp sees the tile
          if (any_valid) {  // (rows past the last token may hold anything)
            uint32_t zero[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) zero[e] = 0u;
            tmem_st32(ts, zero);
            tmem_st32(ts + 32, zero);
          }
          arrive(0, 2);
          ++it;
          ++tiles;
          continue;
        }
        const bool masked = k0 < warp_all_lo || k0 + kTile > warp_all_hi;
        // every key of the tile lies at or before every position of the warp, or at or after them
        const bool before = !BIAS || k0 + kTile - 1 <= pos_min, after = BIAS && k0 >= pos_max;
        const float slope_to = before ? row.slope : -row.slope;
        // the bias (log2) of the nearest of the keys [key, key + n)
        auto near_bias = [&](int key, int n) {
          if (!BIAS) return 0.f;
          const float e = (float)(int)((unsigned)key - (unsigned)row.pos);
          return -row.slope * fmaxf(0.f, fmaxf(e, -(e + (float)(n - 1))));
        };
        // The keys that the guard warp has found: rows that see one are marked (before the last weights are handed over,
        // which lets the tile's results be overwritten).
        auto mark = [&]() {
          const int g = guards - 1, ws = PAIR ? 0 : stream;
          if (!__all_sync(0xffffffffu, mbar_wait_role(sm.vsafe(ws, g), (g / kSafeRing) & 1, fail))) return false;
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            uint32_t bits = s_bad[ws][g % kSafeRing][q];
            while (bits) {
              const int key = k0 + 32 * q + __ffs(bits) - 1;
              bits &= bits - 1;
              bad_row = bad_row || (key >= row.lo && key < row.hi);
            }
          }
          return true;
        };
        // The weights of N columns, packed, and their sum: v holds the scores less the reference.
        auto pack_n = [&](const float* v, uint32_t* w, auto count) {
          constexpr int N = decltype(count)::value;
          uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const float y0 = fast_exp2(v[e]), y1 = fast_exp2(v[e + 1]);
            acc[(e >> 1) & 3] = add_f32x2(acc[(e >> 1) & 3], f32x2(y0, y1));
            w[e >> 1] = pack16<F16>(y0, y1);
          }
          float s0, s1, s2, s3;
          f32x2_split(add_f32x2(acc[0], acc[1]), s0, s1);
          f32x2_split(add_f32x2(acc[2], acc[3]), s2, s3);
          return (s0 + s1) + (s2 + s3);
        };
        auto pack = [&](const auto& v, auto& w) {
          return pack_n(v, w, std::integral_constant<int, sizeof(v) / sizeof(float)>());
        };
        auto load = [&](int col, auto& v) {
          constexpr int N = sizeof(v) / sizeof(float);
#pragma unroll
          for (int q = 0; q < N; q += 32) tmem_ld32(ts + col + q, v + q);
        };
        auto loaded = [](auto& v) {
          tmem_wait_ld(v);
          if constexpr (sizeof(v) == 64 * sizeof(float)) reg_fence(v + 32);
        };
        // The slow path for the N raw scores of columns col ..: masks (by 32 columns, where a row of the warp needs
        // them), the largest score, a moved reference with O rescaled (o_half, o_phase: the last product in O, if any),
        // the weights. False when a wait gave up.
        auto slow_weights = [&](auto& v, auto& w, int col, bool in_o, int o_half, int o_phase) {
          constexpr int N = sizeof(v) / sizeof(float);
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          bool seen[N / 32];  // by some row of the warp
          // The scores are taken less `base`, close to the largest, where that is the fused form's to give: a distance
          // bias of thousands then costs them no bits. Large references of other kinds: see kRefExact.
          float base = ref == -INFINITY ? near_bias(k0 + col, N) : ref;
          if (!(fabsf(base) <= kRefExact)) base = 0.f;
#pragma unroll
          for (int q = 0; q < N; q += 32) {
            const int key = k0 + col + q;
            seen[q / 32] = key < warp_hi && key + 32 > warp_lo;
            if (!seen[q / 32]) continue;
            const bool cut = key < warp_all_lo || key + 32 > warp_all_hi;
            const uint32_t keys = seen_keys(row, key);
            if (CAP && cut) mask_scores(v + q, keys, 0.f);  // (four share a reciprocal)
            row_scores<CAP, BIAS, 32, false>(v + q, sc, row, k0, col + q, base, row.slope);
            if (cut) mask_scores(v + q, keys, -INFINITY);
#pragma unroll
            for (int e = 0; e < 32; e += 2) mx[(e >> 1) & 3] = max3(mx[(e >> 1) & 3], v[q + e], v[q + e + 1]);
          }
          const float largest = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
          const float have = ref - base;  // (relative to the base)
          const float next = largest > have + ref_slack<F16>() ? base + (largest - ref_drop<F16>()) : ref;
          const bool moves = next != ref && ref != -INFINITY;
          if (__any_sync(0xffffffffu, moves)) {
            const float f = moves ? fast_exp2(ref - next) : 1.f;
            if (in_o) {
              if (!__all_sync(0xffffffffu, mbar_wait_role(sm.odone(stream, o_half), o_phase & 1, fail))) return false;
              tcgen05_after_sync();
#pragma unroll 1
              for (int q = 0; q < 8; ++q) {
                float o[16];
                tmem_ld16(to + 16 * q, o);
                tmem_wait_ld16(o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] *= f;
                tmem_st16(to + 16 * q, reinterpret_cast<const uint32_t*>(o));
              }
            }
            sum *= f;
          }
          ref = next;
          careful = __any_sync(0xffffffffu, ref == -INFINITY || fabsf(ref) > kRefExact);
          const float rr = ref == -INFINITY ? 0.f : ref - base;
          const uint64_t r2 = f32x2(-rr, -rr);
#pragma unroll
          for (int q = 0; q < N; q += 32) {
            if (seen[q / 32]) {
#pragma unroll
              for (int e = q; e < q + 32; e += 2) f32x2_split(add_f32x2(f32x2(v[e], v[e + 1]), r2), v[e], v[e + 1]);
              sum += pack_n(v + q, w + q / 2, std::integral_constant<int, 32>());
            } else {
#pragma unroll
              for (int e = 0; e < 16; ++e) w[q / 2 + e] = 0u;
            }
          }
          return true;
        };
        // A row without a reference takes one from 32 columns of its first tile, where no mask is in the way: any finite
        // one will do that the sums do not outgrow, and the fast path checks that.
        if (careful && !masked && __any_sync(0xffffffffu, ref == -INFINITY)) {
          const int col = MODE == kFew ? 32 * (warp & 3) : 0;
          float v[32];
          load(col, v);
          loaded(v);
          const float near = near_bias(k0 + col, 32);
          row_scores<CAP, BIAS, 32, false>(v, sc, row, k0, col, near, row.slope);
          float mx = -INFINITY, mx2 = -INFINITY;
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            mx = max3(mx, v[e], v[e + 1]);
            mx2 = max3(mx2, v[e + 2], v[e + 3]);
          }
          mx = fmaxf(mx, mx2);
          if (ref == -INFINITY && mx > -INFINITY) ref = near + (mx - ref_drop<F16>());
          careful = __any_sync(0xffffffffu, ref == -INFINITY || fabsf(ref) > kRefExact);
        }
        // Fast path: no mask, a reference in every row, the bias linear. Straight-line code, checked by the sum afterwards;
        // nothing is stored before the check.
        const bool bent = !before && !after;
        bool slow = masked || careful || bent;
        if (guarded && !masked) ok = mark();
        if (!ok) break;
        if constexpr (MODE == kFew) {  // this warp's quarter of the keys
          const int quarter = warp & 3, col = 32 * quarter;
          uint32_t w[16], zero[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e] = zero[e] = 0u;
          if (k0 + col < warp_hi && k0 + col + 32 > warp_lo) {
            float v[32];
            load(col, v);
            loaded(v);
            slow = careful || bent || k0 + col < warp_all_lo || k0 + col + 32 > warp_all_hi;
            if (!slow) {
              row_scores<CAP, BIAS, 32, true>(v, sc, row, k0, col, ref, slope_to);
              const float quarter_sum = pack(v, w);
              slow = __any_sync(0xffffffffu, !(quarter_sum <= sum_max<F16>()));
              if (slow) {
                load(col, v);
                loaded(v);
              } else {
                sum += quarter_sum;
              }
            }
            if (slow) ok = slow_weights(v, w, col, it > 0, 1, tiles - 1);
            if (!ok) break;
          }
#pragma unroll
          for (int q = 1; q < 4; ++q) tmem_st16(ts + 16 * ((quarter + q) & 3), zero);
          tmem_st16(ts + 16 * quarter, w);
          if (guarded && masked) ok = mark();
          if (!ok) break;
          arrive(0, 2);
        } else {
          // Each half of a tile is handed over as it is ready, so that its product runs under the next half. Without a
          // cap the second half's arithmetic starts before the first half's hand-over has gone through.
          int first_half = 0;
          if (!CAP && !slow) {
            float v[2][64];
            uint32_t w[2][32];
            load(0, v[0]);
            loaded(v[0]);
            load(64, v[1]);
            row_scores<CAP, BIAS, 64, true>(v[0], sc, row, k0, 0, ref, slope_to);
            const float sum0 = pack(v[0], w[0]);
            slow = __any_sync(0xffffffffu, !(sum0 <= sum_max<F16>()));  // a reference is too low (or a score NaN)
            if (!slow) {
              sum += sum0;
              first_half = 1;
              tmem_st32(ts, w[0]);
              loaded(v[1]);
              row_scores<CAP, BIAS, 64, true>(v[1], sc, row, k0, 64, ref, slope_to);
              arrive(0, 1);
              const float sum1 = pack(v[1], w[1]);
              slow = __any_sync(0xffffffffu, !(sum1 <= sum_max<F16>()));
              if (!slow) {
                sum += sum1;
                tmem_st32(ts + 32, w[1]);
                arrive(1, 1);
              }
            } else {
              loaded(v[1]);
            }
          }
          if (CAP || slow) {
#pragma unroll 1
            for (int half = first_half; half < 2; ++half) {
              float v[64];
              uint32_t w[32];
              bool slow_half = slow || careful;
              load(64 * half, v);
              loaded(v);
              if (CAP && !slow_half) {
                row_scores<CAP, BIAS, 64, true>(v, sc, row, k0, 64 * half, ref, slope_to);
                const float half_sum = pack(v, w);
                slow_half = __any_sync(0xffffffffu, !(half_sum <= sum_max<F16>()));
                if (slow_half) {
                  load(64 * half, v);
                  loaded(v);
                } else {
                  sum += half_sum;
                }
              }
              if (slow_half) ok = slow_weights(v, w, 64 * half, it + half > 0, half ^ 1, half ? tiles : tiles - 1);
              if (!ok) break;
              tmem_st32(ts + 32 * half, w);  // (over columns of S that both halves have left)
              if (half == 1 && guarded && masked) {
                ok = mark();
                if (!ok) break;
              }
              arrive(half, 1);
            }
          }
        }
        if (!ok) break;
        ++it;
        ++tiles;
      }
      // where the row goes; the next item's row is asked for before this one is written
      const size_t out_row = ((size_t)x.b * a.tq + token) * a.heads_q + head;
      const bool whole = !p.shares;
      const long long part_at = (long long)x.slot * L::kItemRows + (PAIR ? stream * kTile : 0) + r;
      char* dst = whole ? static_cast<char*>(a.out) +
                              (x.b * a.o_b + head * a.o_h + token * a.o_t) * (p.out_f32 ? 4 : 2)
                        : reinterpret_cast<char*>(p.part_o + part_at * kHeadDim);
      const long long stat_at = whole ? x.b * a.s_b + head * a.s_h + token * a.s_t : part_at;
      const int n = x.n, set = x.b, head0 = x.h * a.G, slot = x.slot;
      if (ok) ok = next_item(round + 1, x);
      if (ok && x.valid) load_row();
      if (ok && it > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait_role(sm.odone(stream, 1), (tiles - 1) & 1, fail));
        tcgen05_after_sync();
      }
      // Output. kPair: each thread its row of O. kOne: the streams hold two parts of the same rows, in the same TMEM
      // lanes; each warpgroup joins one half of the channels. kFew: eight parts, joined through shared memory.
      if constexpr (!PAIR) {
        s_part[part][0][r] = it > 0 ? ref : -INFINITY;
        s_part[part][1][r] = it > 0 ? sum : 0.f;
        s_mark[part][r] = bad_row;
        tcgen05_before_sync();
        if (softmax_sync(!ok || *fail)) break;  // (both streams' products are done)
        tcgen05_after_sync();
      } else if (!ok) {
        break;
      }
      // A row's parts taken together: the largest reference, log2 of the sum, factors of the parts (times 2^(reference of
      // the part - top)) and of the request's own output.
      struct Joined {
        float top, lse2, f0, f1;
      };
      auto join = [&](int row_in_tile, bool there, size_t at_row) {
        Joined q;
        float total = sum;
        bool marked = bad_row;
        q.top = ref;
        if constexpr (!PAIR) {
          q.top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 2 * L::kCopies; ++i) q.top = fmaxf(q.top, s_part[i][0][row_in_tile]);
          total = 0.f;
          marked = false;
#pragma unroll
          for (int i = 0; i < 2 * L::kCopies; ++i) {
            const float g = q.top == -INFINITY ? 0.f : fast_exp2(s_part[i][0][row_in_tile] - q.top);
            total = fmaf(s_part[i][1][row_in_tile], g, total);
            marked = marked || s_mark[i][row_in_tile];
          }
        }
        q.lse2 = total == 0.f ? -INFINITY : q.top + log2f(total);
        q.f0 = total == 0.f ? 0.f : 1.f / total;
        q.f1 = 0.f;
        if (whole && a.own_out && there) join_own(a, at_row, q.lse2, q.f0, q.f1);
        if (marked) q.f0 = __int_as_float(0x7fffffff);
        return q;
      };
      const Joined jn = join(r, valid, out_row);
      // (a row whose sum is 0 has seen nothing, or only scores of -inf: its O holds zeros or, never written, anything)
      const bool blank = jn.f0 == 0.f;
      const float f1 = jn.f1;
      auto part_factor = [&](int i) { return jn.f0 * (jn.top == -INFINITY ? 0.f : fast_exp2(s_part[i][0][r] - jn.top)); };
      if constexpr (MODE == kFew) {
        // 8 rows and 64 channels at a time: every part scaled into shared memory, then summed (thread: two channels of the
        // row `warp` of the eight). Few rows, few rounds: one decoded token's take two.
        float* ex = reinterpret_cast<float*>(smem_raw + (sm.exchange() - smem_u32(smem_raw)));
        const float g = blank || it == 0 ? 0.f : part_factor(part);
        const bool f32 = !whole || p.out_f32;
#pragma unroll 1
        for (int row0 = 0; row0 < a.tq * a.G; row0 += 8) {
          const int orow = row0 + warp, otoken = orow >> p.log2_G, ohead = head0 + (orow & (a.G - 1));
          const bool othere = otoken < a.tq;
          const size_t orow_out = ((size_t)set * a.tq + otoken) * a.heads_q + ohead;
          const Joined jo = join(orow, othere, orow_out);
          char* odst = whole ? static_cast<char*>(a.out) +
                                   (set * a.o_b + ohead * a.o_h + otoken * a.o_t) * (p.out_f32 ? 4 : 2)
                             : reinterpret_cast<char*>(p.part_o + ((size_t)slot * L::kItemRows + orow) * kHeadDim);
#pragma unroll 1
          for (int ch0 = 0; ch0 < kHeadDim; ch0 += 64) {
            float v[64];
            if (it > 0) {
              tmem_ld32(to + ch0, v);
              tmem_ld32(to + ch0 + 32, v + 32);
              tmem_wait_ld(v);
              reg_fence(v + 32);
            }
            if ((lane & 24) == row0) {
              float4* mine = reinterpret_cast<float4*>(ex + (part * 8 + (lane & 7)) * kExPitch);
#pragma unroll
              for (int e = 0; e < 64; e += 4)
                mine[e / 4] = g != 0.f ? make_float4(v[e] * g, v[e + 1] * g, v[e + 2] * g, v[e + 3] * g)
                                       : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            softmax_sync(false);
            if (othere) {
              float y0 = 0.f, y1 = 0.f;
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float2 z = *reinterpret_cast<const float2*>(ex + (i * 8 + warp) * kExPitch + 2 * lane);
                y0 += z.x;
                y1 += z.y;
              }
              const int ch = ch0 + 2 * lane;
              if (jo.f1 != 0.f) {
                const float2 o = *reinterpret_cast<const float2*>(a.own_out + orow_out * kHeadDim + ch);
                y0 = fmaf(o.x, jo.f1, y0);
                y1 = fmaf(o.y, jo.f1, y1);
              }
              if (f32)
                reinterpret_cast<float2*>(odst)[ch / 2] = make_float2(y0, y1);
              else
                reinterpret_cast<uint32_t*>(odst)[ch / 2] = pack16<F16>(y0, y1);
            }
            softmax_sync(false);
          }
          if (othere && lane == 0) {
            if (whole)
              store_stat(a, set * a.s_b + ohead * a.s_h + otoken * a.s_t, jo.lse2);
            else
              p.part_lse[(size_t)slot * L::kItemRows + orow] = jo.lse2;
          }
        }
        tcgen05_before_sync();
        if (softmax_sync(*fail)) break;
        continue;
      }
      const float lse2 = jn.lse2;
      const float g0 = PAIR ? jn.f0 : part_factor(0), g1 = PAIR ? 0.f : part_factor(1);
      const uint32_t o0 = PAIR ? to : tmem + 256 + lanes;
      const bool has0 = PAIR ? it > 0 : n > 0, has1 = !PAIR && n > 1;
      const float* own = a.own_out + out_row * kHeadDim;
#pragma unroll 1
      for (int q = 0; q < (PAIR ? 4 : 2); ++q) {
        const int ch = 32 * (PAIR ? q : 2 * stream + q);
        float v[32];
        if (has0) {
          tmem_ld32(o0 + ch, v);
          tmem_wait_ld(v);
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = blank || !has0 ? 0.f : v[e] * g0;
        if (has1) {
          float v1[32];
          tmem_ld32(o0 + 128 + ch, v1);
          tmem_wait_ld(v1);
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = blank ? 0.f : fmaf(v1[e], g1, v[e]);
        }
        if (valid) {
          if (f1 != 0.f) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 o = *reinterpret_cast<const float4*>(own + ch + e);
              v[e] = fmaf(o.x, f1, v[e]);
              v[e + 1] = fmaf(o.y, f1, v[e + 1]);
              v[e + 2] = fmaf(o.z, f1, v[e + 2]);
              v[e + 3] = fmaf(o.w, f1, v[e + 3]);
            }
          }
          store_out32<F16>(dst, !whole || p.out_f32, ch, v);
        }
      }
      if (valid && (PAIR || stream == 0)) {
        if (whole)
          store_stat(a, stat_at, lse2);
        else
          p.part_lse[stat_at] = lse2;
      }
      if constexpr (!PAIR) {  // both warpgroups have read both O before the next item's products overwrite them
        tcgen05_before_sync();
        if (softmax_sync(*fail)) break;
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

template <bool F16, int MODE>
cudaError_t launch_variant(const FlashKernelArgs& p, int grid, cudaStream_t st) {
  const bool cap = p.a.softcap > 0.f, bias = p.a.slopes != nullptr;
  auto k = cap ? (bias ? flash_kernel<F16, MODE, true, true> : flash_kernel<F16, MODE, true, false>)
               : (bias ? flash_kernel<F16, MODE, false, true> : flash_kernel<F16, MODE, false, false>);
  static std::atomic<uint64_t> configured[4];  // per variant: one bit per device
  std::atomic<uint64_t>& done = configured[2 * cap + bias];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev > 63 || !(done.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<MODE>::kSmem);
    if (e != cudaSuccess) return e;
    done.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_chained(k, dim3(grid), dim3(kThreads), Layout<MODE>::kSmem, st, p);
}

}  // namespace flash
}  // namespace mikv
