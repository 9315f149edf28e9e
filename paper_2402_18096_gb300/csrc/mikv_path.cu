// mikv_path.cu — what follows the attention of drafted tokens: the importance that an accepted path hands out, its entry
// into the cache with the demotions that follow, and copies of whole requests.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "mikv_quant_rows.cuh"
#include "mikv_rows.cuh"
#include "mikv_tree.h"

namespace mikv {
namespace {

// Accepted nodes of a request, by every thread of a block of at least kTreeNodes threads: their number; nodes in
// `path` (shared). The entries end at the first that is no node.
__device__ __forceinline__ int accepted(const int32_t* entries, int steps, int nodes, int* path, int* count) {
  const int i = threadIdx.x;
  if (i == 0) *count = steps;
  __syncthreads();
  if (i < steps) {
    const int x = entries[i];
    path[i] = x;
    if (x < 0 || x >= nodes) atomicMin(count, i);
  }
  __syncthreads();
  return *count;
}

// acc and gained on mma.sync: a warp holds 16 keys as the A operand, straight from memory (a lane's 16 bytes of a key are the
// k elements of two steps, in an order that the queries share), and goes through the path's rows (node, query head) 16
// columns at a time. Bound by the keys' bytes (256 a slot): every key is read once, whatever the path's length, and
// nothing is staged on its way; the rows are staged kRowChunk at a time, once where they fit. Block (x, bh): x < gridDim.x -
// 1 takes key blocks x, x + gridDim.x - 1, ..., the next one's keys on their way under the products of this; the last one
// the path's own nodes. 256 KV heads of 6554 slots at most, 20 rows at most: 69 us with one block of 256 keys to a CTA, whose
// start every one of them waited for, 47 here (4.4 TB/s, 65 % of a copy).
constexpr int kImpWarps = 8, kBlockKeys = kImpWarps * 16, kRowChunk = 64, kRowPitch = 2 * kHeadDim + 16;
__global__ void __launch_bounds__(32 * kImpWarps, 2) importance_kernel(float* acc, const __nv_bfloat16* k_hi,
                                                                      const PathArgs a, int Hq, int Hkv, int hi_stride) {
  __shared__ int path[kTreeNodes], count;
  __shared__ __align__(16) uint8_t s_q[kRowChunk * kRowPitch];
  __shared__ float s_lse[kRowChunk];  // log2; +inf where a row weighs nothing
  const int bh = blockIdx.y, b = bh / Hkv, h = bh - b * Hkv, G = Hq / Hkv, log2_G = 31 - __clz(G);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  grid_dependency_wait();
  allow_dependent_launch();
  const bool slots = blockIdx.x + 1 < gridDim.x;
  const int stride = slots ? (gridDim.x - 1) * kBlockKeys : kBlockKeys, n_hi = a.held.hi(b);
  int first = slots ? blockIdx.x * kBlockKeys : 0, last = n_hi;
  if (slots && first >= last) return;
  // a block's keys of this warp: rows g and g + 8; four chunks of 16 bytes of each
  uint4 key[2][4], next[2][4];
  auto load = [&](int at, uint4 (&to)[2][4]) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int s = min(at + 16 * warp + 8 * r + g, last - 1);
      const __nv_bfloat16* row = slots ? k_hi + ((size_t)bh * hi_stride + s) * kHeadDim
                                       : static_cast<const __nv_bfloat16*>(a.k.p) + b * a.k.b + h * a.k.h + path[s] * a.k.t;
#pragma unroll
      for (int c = 0; c < 4; ++c) to[r][c] = __ldg(reinterpret_cast<const uint4*>(row + 32 * c) + t);
    }
  };
  if (slots) load(first, key);
  const int n = accepted(a.path + (size_t)b * a.steps, a.steps, a.nodes, path, &count);
  float* gained = a.gained + (size_t)bh * a.steps;
  if (!slots && threadIdx.x < a.steps && (int)threadIdx.x >= n) gained[threadIdx.x] = 0.f;
  if (n == 0) return;
  if (!slots) {
    last = n;
    load(0, key);
  }
  const int free_slot = slots ? a.held.free_slot(bh, n_hi) : -1;
  float* to = slots ? acc + (size_t)bh * hi_stride : gained;
  constexpr float kLog2e = 1.4426950408889634f;
  const float scale = a.sm_scale * kLog2e;
  const int rows = n << log2_G;
  bool staged = false;
#pragma unroll 1
  for (; first < last; first += stride) {
    if (first + stride < last) load(first + stride, next);
    const int mine = first + 16 * warp;
    float sum[2] = {0.f, 0.f}, old[2] = {0.f, 0.f};
    bool writes[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int s = mine + 8 * k + g;
      writes[k] = t == 0 && s < last && s != free_slot;
      if (slots && writes[k]) old[k] = to[s];
    }
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += kRowChunk) {
      const int here = min(kRowChunk, rows - r0), padded = (here + 15) & ~15;
      if (!staged) {
        __syncthreads();
        for (int i = threadIdx.x; i < padded * 16; i += 32 * kImpWarps) {
          const int r = i >> 4, c = i & 15, node = path[min((r0 + r) >> log2_G, n - 1)], j = h * G + ((r0 + r) & (G - 1));
          uint4 x = make_uint4(0u, 0u, 0u, 0u);
          if (r < here)
            x = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + j * a.q.h + node * a.q.t) + c);
          *reinterpret_cast<uint4*>(s_q + r * kRowPitch + 16 * c) = x;
          if (c == 0) {
            const float e = r < here ? a.lse[((size_t)b * Hq + j) * a.nodes + node] : INFINITY;
            s_lse[r] = isinf(e) ? INFINITY : e * kLog2e;
          }
        }
        __syncthreads();
        staged = rows <= kRowChunk;
      }
      if (mine >= last) continue;
#pragma unroll 1
      for (int col = 0; col < padded; col += 16) {
        float d[2][4] = {};
#pragma unroll
        for (int c = 0; c < 4; ++c) {  // steps 2 c and 2 c + 1
          const uint4 x = key[0][c], y = key[1][c];
          const uint32_t a0[4] = {x.x, y.x, x.y, y.y}, a1[4] = {x.z, y.z, x.w, y.w};
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4 q = *reinterpret_cast<const uint4*>(s_q + (col + 8 * i + g) * kRowPitch + 64 * c + 16 * t);
            mma_bf16(d[i], a0, q.x, q.y);
            mma_bf16(d[i], a1, q.z, q.w);
          }
        }
        // columns 2 t and 2 t + 1 of this lane; a path's own node receives from itself and the later ones
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = col + 8 * i + 2 * t + e, step = slots ? INT_MAX : (r0 + r) >> log2_G;
            const float lse = s_lse[r];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const bool sees = lse != INFINITY && step >= mine + 8 * k + g;
              sum[k] += sees ? fast_exp2(fmaf(d[i][2 * k + e], scale, -lse)) : 0.f;
            }
          }
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float x = sum[k];
      x += __shfl_xor_sync(0xffffffffu, x, 1);
      x += __shfl_xor_sync(0xffffffffu, x, 2);
      if (writes[k]) to[mine + 8 * k + g] = old[k] + x;
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) key[r][c] = next[r][c];
  }
}

// What a commit does to the lengths of a request.
struct Commit {
  int n_hi, n_lo, count, gone;  // in use before; accepted; demoted
  bool fits;
};
__device__ __forceinline__ Commit commit_of(const PathArgs& a, int b, int count, int bits, int lo_cap) {
  Commit c;
  c.n_hi = a.held.hi(b);
  c.n_lo = bits ? a.held.lo(b) : 0;
  const int free_slots = a.held.slots ? 1 : 0;
  c.count = c.n_hi > 0 ? count : 0;
  c.gone = max(0, c.n_hi - free_slots + c.count - (a.held.hi_cap - free_slots));
  if (c.count == 0) c.gone = 0;
  c.fits = bits == 0 || c.n_lo + c.gone <= lo_cap;
  return c;
}

__device__ __forceinline__ void write_lengths(const PathArgs& a, int b, const Commit& m, int bits) {
  const int count = m.fits ? m.count : 0, gone = m.fits ? m.gone : 0;
  if (a.n_hi_out) a.n_hi_out[b] = m.n_hi + count - gone;
  if (a.n_lo_out) a.n_lo_out[b] = m.n_lo + (bits ? gone : 0);
  if (a.next) a.next[b] = a.first[b] + count;
}

struct CommitArrays {
  __nv_bfloat16 *k_hi, *v_hi;
  int32_t* hi_tok;
  float* acc;
  uint8_t *k_codes, *v_codes;
  __half2 *k_params, *v_params;
  int32_t* lo_tok;
  const float* balancer;
  int Hkv, hi_stride, lo_cap;
};

// One block per KV head. The demoted entries are found one after another, the least (score, id, place) of those left
// (places: the slots, then the path's nodes); a warp to a row quantizes them; then the tokens that stay are written. Bound
// by latency: a demotion costs two reductions, and the rows of all demotions are in flight together. The scores and ids of
// the first 2048 entries are read once and stay in registers (kOwn entries a thread); those behind are read again, from
// L2, for every demotion. Eight demotions, us a call in a graph: 64 requests of up to 1025 slots, 32 KV heads 9.7; 32 of 2001, 8
// KV heads 14.7, of 6555 33.6 (one demotion 10.9).
constexpr int kCommitThreads = 256, kOwn = 8;
template <int BITS, int GROUP>
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const CommitArrays c, const PathArgs a, bool lengths) {
  __shared__ int path[kTreeNodes], count, victim[kTreeNodes], place[kTreeNodes];
  __shared__ unsigned long long s_key[kCommitThreads / 32];
  __shared__ int s_at[kCommitThreads / 32];
  const int bh = blockIdx.x, b = bh / c.Hkv, h = bh - b * c.Hkv, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dependency_wait();
  allow_dependent_launch();
  const Commit m = commit_of(a, b, accepted(a.path + (size_t)b * a.steps, a.steps, a.nodes, path, &count), BITS, c.lo_cap);
  if (lengths && h == 0 && tid == 0) write_lengths(a, b, m, BITS);
  if (m.count == 0) return;
  const int free_slot = a.held.free_slot(bh, m.n_hi);
  if (!m.fits || (a.held.slots && free_slot < 0)) {
    if (tid == 0) record_error(a.status, kErrBounds);
    return;
  }
  const size_t hi0 = (size_t)bh * c.hi_stride;
  const int entries = m.n_hi + m.count, tok0 = a.first[b];
  const float* gained = a.gained + (size_t)bh * a.steps;
  auto key_of = [&](int e) {
    return e < m.n_hi ? order_key(c.acc[hi0 + e], c.hi_tok[hi0 + e]) : order_key(gained[e - m.n_hi], tok0 + e - m.n_hi);
  };
  unsigned long long own[kOwn];  // entries tid, tid + kCommitThreads, ...; the highest key: none
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int e = tid + i * kCommitThreads;
    own[i] = m.gone > 0 && e < entries && e != free_slot ? key_of(e) : ~0ull;
  }
  unsigned long long last_key = 0ull;  // the least entry found so far
  int last_at = -1;
  for (int j = 0; j < m.gone; ++j) {
    unsigned long long best = ~0ull;
    int at = entries;
    auto consider = [&](unsigned long long k, int e) {
      const bool left = j == 0 || k > last_key || (k == last_key && e > last_at);
      if (left && (at == entries || k < best)) best = k, at = e;
    };
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const int e = tid + i * kCommitThreads;
      if (e < entries && e != free_slot) consider(own[i], e);
    }
    for (int e = tid + kOwn * kCommitThreads; e < entries; e += kCommitThreads)
      if (e != free_slot) consider(key_of(e), e);
    auto reduce = [&]() {
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) {
        const unsigned long long k = __shfl_xor_sync(0xffffffffu, best, off);
        const int e = __shfl_xor_sync(0xffffffffu, at, off);
        if (k < best || (k == best && e < at)) best = k, at = e;
      }
    };
    reduce();
    if (lane == 0) s_key[warp] = best, s_at[warp] = at;
    __syncthreads();
    constexpr int W = kCommitThreads / 32;
    best = s_key[lane & (W - 1)], at = s_at[lane & (W - 1)];
    reduce();
    last_key = best, last_at = at;
    if (tid == 0) victim[j] = at;
    __syncthreads();
  }
  if (tid == 0) {  // where the path's nodes go: -1 demoted, else the slot
    for (int i = 0; i < m.count; ++i) place[i] = 0;
    for (int j = 0; j < m.gone; ++j)
      if (victim[j] >= m.n_hi) place[victim[j] - m.n_hi] = -1;
    int j = 0, fresh = m.n_hi;
    for (int i = 0; i < m.count; ++i) {
      if (place[i] < 0) continue;
      while (j < m.gone && victim[j] >= m.n_hi) ++j;
      place[i] = j < m.gone ? victim[j++] : fresh++;
    }
  }
  __syncthreads();
  auto node_row = [&](const TreeView& x, int i) {
    return static_cast<const __nv_bfloat16*>(x.p) + b * x.b + h * x.h + path[i] * x.t;
  };
  if constexpr (BITS != 0) {
    for (int x = warp; x < 2 * m.gone; x += kCommitThreads / 32) {
      const int j = x >> 1, e = victim[j];
      const bool val = x & 1;
      const __nv_bfloat16* src = e < m.n_hi ? (val ? c.v_hi : c.k_hi) + (hi0 + e) * kHeadDim
                                            : node_row(val ? a.v : a.k, e - m.n_hi);
      const size_t row = (size_t)bh * c.lo_cap + m.n_lo + j;
      quantize_row_warp<BITS, GROUP>(src, val || !c.balancer ? nullptr : c.balancer + h * kHeadDim,
                                     (val ? c.v_codes : c.k_codes) + row * 16 * BITS,
                                     (val ? c.v_params : c.k_params) + row * (kHeadDim / GROUP), lane);
      if (!val && lane == 0) c.lo_tok[row] = e < m.n_hi ? c.hi_tok[hi0 + e] : tok0 + e - m.n_hi;
    }
    __syncthreads();
  }
  for (int x = warp; x < 2 * m.count; x += kCommitThreads / 32) {
    const int i = x >> 1, to = place[i];
    const bool val = x & 1;
    if (to < 0) continue;
    reinterpret_cast<uint2*>((val ? c.v_hi : c.k_hi) + (hi0 + to) * kHeadDim)[lane] =
        reinterpret_cast<const uint2*>(node_row(val ? a.v : a.k, i))[lane];
    if (!val && lane == 0) {
      c.hi_tok[hi0 + to] = tok0 + i;
      c.acc[hi0 + to] = gained[i];
    }
  }
}

// The lengths after a commit, where they are written over those that it reads: a launch of its own.
__global__ void __launch_bounds__(kTreeNodes) commit_lengths_kernel(const PathArgs a, int bits, int lo_cap) {
  __shared__ int path[kTreeNodes], count;
  const int b = blockIdx.x;
  grid_dependency_wait();
  allow_dependent_launch();
  const Commit m = commit_of(a, b, accepted(a.path + (size_t)b * a.steps, a.steps, a.nodes, path, &count), bits, lo_cap);
  if (threadIdx.x == 0) write_lengths(a, b, m, bits);
}

// Copies. An array of a cache, and which of a request's rows it keeps.
enum RowKind { kHiRows, kLoRows, kStagedRows, kGroups };
struct CopyArray {
  const char* from;
  char* to;
  int from_cap, to_cap;  // rows per head
  int from_row, to_row;  // first row
  int row_bytes, kind;
};
constexpr int kCopyArrays = 16, kCopyPairs = 256, kCopyThreads = 256, kInFlight = 8;
struct CopyArgs {
  CopyArray x[kCopyArrays];
  int2 pair[kCopyPairs];
  CopyLengths len;
  int arrays, heads, hi_cap, kch, chunk;
};

// Block (pair, chunk, head): its chunk of the bytes that the request keeps of this head, array after array. Pairs run
// fastest, so that those of one source read it from L2. Long requests are bound by HBM (16 copies of up to 8192 tokens, 40
// heads: 114 us, 82 % of a copy), short ones by the way through nine arrays (three of 512 tokens, 32 heads: 14.6 us in a
// graph, 2.3 at a copy's rate).
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyArgs a) {
  const int2 pair = a.pair[blockIdx.x];
  grid_dependency_wait();
  allow_dependent_launch();
  const int h = blockIdx.z;
  const int n_hi = a.len.n_hi ? max(0, min(a.len.n_hi[pair.x], a.hi_cap)) : a.hi_cap;
  const int n_lo = a.len.n_lo ? max(0, min(a.len.n_lo[pair.x], a.len.n_lo_max)) : a.len.n_lo_max;
  if (blockIdx.y == 0 && threadIdx.x == 0) {
    if (a.len.to_slots) a.len.to_slots[pair.y * a.heads + h] = a.len.slots[pair.x * a.heads + h];
    if (h == 0 && a.len.to_n_hi) a.len.to_n_hi[pair.y] = n_hi;
    if (h == 0 && a.len.to_n_lo) a.len.to_n_lo[pair.y] = n_lo;
  }
  const int kept = a.kch ? n_lo / kKchGroup * kKchGroup : n_lo;
  for (int chunk = blockIdx.y;; chunk += gridDim.y) {
    long long begin = (long long)chunk * a.chunk, end = begin + a.chunk;
    for (int i = 0; i < a.arrays && end > 0; ++i) {
      const CopyArray& x = a.x[i];
      const int rows = x.kind == kHiRows ? n_hi : x.kind == kLoRows ? kept : x.kind == kGroups ? kept / kKchGroup : n_lo - kept;
      const long long bytes = (long long)rows * x.row_bytes;
      const long long lo = max(begin, 0ll), hi = min(end, bytes);
      const char* from = x.from + (((size_t)pair.x * a.heads + h) * x.from_cap + x.from_row) * x.row_bytes;
      char* to = x.to + (((size_t)pair.y * a.heads + h) * x.to_cap + x.to_row) * x.row_bytes;
      // (ids and scores of staged rows may begin anywhere)
      const bool wide = ((reinterpret_cast<uintptr_t>(from) | reinterpret_cast<uintptr_t>(to)) & 15) == 0;
      const long long end16 = wide ? lo + ((hi - lo) & ~15ll) : lo;
      long long at = lo + 16 * threadIdx.x;
      for (; at < end16; at += 16ll * kCopyThreads * kInFlight) {
        uint4 v[kInFlight];
#pragma unroll
        for (int k = 0; k < kInFlight; ++k)
          if (at + 16ll * kCopyThreads * k < end16) v[k] = __ldg(reinterpret_cast<const uint4*>(from + at + 16ll * kCopyThreads * k));
#pragma unroll
        for (int k = 0; k < kInFlight; ++k)
          if (at + 16ll * kCopyThreads * k < end16) __stcs(reinterpret_cast<uint4*>(to + at + 16ll * kCopyThreads * k), v[k]);
      }
      for (at = end16 + 4 * threadIdx.x; at < hi; at += 4 * kCopyThreads)
        *reinterpret_cast<uint32_t*>(to + at) = *reinterpret_cast<const uint32_t*>(from + at);
      const long long whole = (bytes + 15) / 16 * 16;  // (the next array's pieces begin at a multiple of 16 bytes)
      begin -= whole;
      end -= whole;
    }
    if (begin >= 0) break;  // past the last array
  }
}

}  // namespace

cudaError_t launch_path_importance(const mikv_shape& s, const PathArgs& a, cudaStream_t st) {
  // a CTA takes 16 key blocks, fewer where that would leave SMs idle (4: 58 us, 8: 50, 16: 47, 26: 48)
  const int blocks = (s.hi_cap + kBlockKeys - 1) / kBlockKeys, heads = s.batch * s.heads_kv;
  const int ctas = std::min(blocks, std::max((blocks + 15) / 16, (4 * 152 + heads - 1) / heads));
  const dim3 grid(ctas + 1, heads);
  return launch_chained(importance_kernel, grid, dim3(32 * kImpWarps), 0, st, a.cache->acc,
                        static_cast<const __nv_bfloat16*>(a.cache->k_hi), a, s.heads_q, s.heads_kv, s.hi_stride);
}

cudaError_t launch_commit(const mikv_shape& s, const PathArgs& a, cudaStream_t st) {
  const mikv_cache& k = *a.cache;
  const CommitArrays c = {static_cast<__nv_bfloat16*>(k.k_hi), static_cast<__nv_bfloat16*>(k.v_hi), k.hi_tok, k.acc,
                          static_cast<uint8_t*>(k.k_codes), static_cast<uint8_t*>(k.v_codes),
                          static_cast<__half2*>(k.k_params), static_cast<__half2*>(k.v_params), k.lo_tok, k.balancer,
                          s.heads_kv, s.hi_stride, s.lo_cap};
  void (*kernel)(const CommitArrays, const PathArgs, bool) = nullptr;
  const bool over = (a.n_hi_out && a.n_hi_out == a.held.n_hi) || (a.n_lo_out && a.n_lo_out == a.held.n_lo) || (a.next && a.next == a.first);
  switch (s.bits == 0 ? 0 : 1000 * s.bits + s.group) {
    case 0: kernel = commit_kernel<0, 32>; break;
    case 2032: kernel = commit_kernel<2, 32>; break;
    case 2064: kernel = commit_kernel<2, 64>; break;
    case 2128: kernel = commit_kernel<2, 128>; break;
    case 3032: kernel = commit_kernel<3, 32>; break;
    case 3064: kernel = commit_kernel<3, 64>; break;
    case 3128: kernel = commit_kernel<3, 128>; break;
    case 4032: kernel = commit_kernel<4, 32>; break;
    case 4064: kernel = commit_kernel<4, 64>; break;
    case 4128: kernel = commit_kernel<4, 128>; break;
    default: return cudaErrorInvalidValue;
  }
  const cudaError_t e = launch_chained(kernel, dim3(s.batch * s.heads_kv), dim3(kCommitThreads), 0, st, c, a, !over);
  if (e != cudaSuccess || !over) return e;
  return launch_chained(commit_lengths_kernel, dim3(s.batch), dim3(kTreeNodes), 0, st, a, s.bits, s.lo_cap);
}

cudaError_t launch_copy_requests(const mikv_shape& s, const mikv_cache& c, const mikv_shape& ts, const mikv_cache& tc,
                                 const int32_t* pairs, int n, const CopyLengths& len, cudaStream_t st) {
  CopyArgs a = {};
  long long most = 0;  // bytes of a request of the longest lengths, per head
  auto add = [&](const void* from, void* to, int from_cap, int to_cap, int from_row, int to_row, int row_bytes, int kind,
                 long long rows) {
    a.x[a.arrays++] = {static_cast<const char*>(from), static_cast<char*>(to), from_cap, to_cap, from_row, to_row,
                       row_bytes, kind};
    most += (rows * row_bytes + 15) / 16 * 16;
  };
  const int hb = hi_bits_of(s), hi_row = hb == 16 ? 2 * kHeadDim : 16 * hb;
  auto add_hi = [&](int from_row, int to_row, int kind, long long rows) {
    add(c.k_hi, tc.k_hi, s.hi_stride, ts.hi_stride, from_row, to_row, hi_row, kind, rows);
    add(c.v_hi, tc.v_hi, s.hi_stride, ts.hi_stride, from_row, to_row, hi_row, kind, rows);
    add(c.hi_tok, tc.hi_tok, s.hi_stride, ts.hi_stride, from_row, to_row, 4, kind, rows);
    add(c.acc, tc.acc, s.hi_stride, ts.hi_stride, from_row, to_row, 4, kind, rows);
  };
  add_hi(0, 0, kHiRows, s.hi_cap);
  if (hb != 16) {
    const int row = 4 * (kHeadDim / kHiGroup);
    add(c.k_hi_params, tc.k_hi_params, s.hi_stride, ts.hi_stride, 0, 0, row, kHiRows, s.hi_cap);
    add(c.v_hi_params, tc.v_hi_params, s.hi_stride, ts.hi_stride, 0, 0, row, kHiRows, s.hi_cap);
  }
  a.kch = kch_of(s);
  if (!evicting(s)) {
    const int row = 4 * (kHeadDim / s.group);
    const long long rows = len.n_lo_max;
    add(c.k_codes, tc.k_codes, s.lo_cap, ts.lo_cap, 0, 0, 16 * s.bits, kLoRows, rows);
    add(c.v_codes, tc.v_codes, s.lo_cap, ts.lo_cap, 0, 0, 16 * s.bits, kLoRows, rows);
    if (a.kch)
      add(c.k_params, tc.k_params, s.lo_cap / kKchGroup, ts.lo_cap / kKchGroup, 0, 0, 4 * kHeadDim, kGroups,
          rows / kKchGroup);
    else
      add(c.k_params, tc.k_params, s.lo_cap, ts.lo_cap, 0, 0, row, kLoRows, rows);
    add(c.v_params, tc.v_params, s.lo_cap, ts.lo_cap, 0, 0, row, kLoRows, rows);
    add(c.lo_tok, tc.lo_tok, s.lo_cap, ts.lo_cap, 0, 0, 4, kLoRows, rows);
    if (a.kch) add_hi(s.hi_cap, ts.hi_cap, kStagedRows, kKchGroup);
  }
  a.len = len;
  a.heads = s.heads_kv;
  a.hi_cap = s.hi_cap;
  // Pieces of 32 KB (what a block has in flight) to 128 KB: enough of them for every SM, and few of them empty where
  // requests are shorter than the caches allow. 8 requests of 20 .. 8192 tokens, twice each: 32 KB 290 us, 128 KB 114.
  const long long share = most * s.heads_kv * std::min(n, kCopyPairs) / (8 * 152);
  a.chunk = (int)std::min(std::max(share & ~32767ll, 32768ll), 131072ll);
  const int chunks = (int)std::min(std::max(1ll, (most + a.chunk - 1) / a.chunk), 65535ll);
  for (int first = 0; first < n; first += kCopyPairs) {
    const int count = std::min(kCopyPairs, n - first);
    for (int i = 0; i < count; ++i) a.pair[i] = make_int2(pairs[2 * (first + i)], pairs[2 * (first + i) + 1]);
    const cudaError_t e = launch_chained(copy_kernel, dim3(count, chunks, s.heads_kv), dim3(kCopyThreads), 0, st, a);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace mikv
