// mikv_path.cu — what follows the attention of drafted tokens: the importance that an accepted path hands out, its entry
// into the cache with the demotions that follow, and copies of whole requests.
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

// acc and gained. Block (x, bh): x < gridDim.x - 1 takes kSlots slots, the last one the path's own nodes; a key to a warp
// at a time, the path's queries in turn.
constexpr int kSlots = 64;
__global__ void __launch_bounds__(256) importance_kernel(float* acc, const __nv_bfloat16* k_hi, const PathArgs a, int Hq,
                                                         int Hkv, int hi_stride) {
  __shared__ int path[kTreeNodes], count;
  const int bh = blockIdx.y, b = bh / Hkv, h = bh - b * Hkv, G = Hq / Hkv, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = accepted(a.path + (size_t)b * a.steps, a.steps, a.nodes, path, &count);
  const bool slots = blockIdx.x + 1 < gridDim.x;
  const int n_hi = a.held.hi(b), free_slot = a.held.free_slot(bh, n_hi);
  const int first = slots ? blockIdx.x * kSlots : 0, last = slots ? min(n_hi, first + kSlots) : a.steps;
  for (int s = first + warp; s < last; s += 8) {
    if (slots && (s == free_slot || n == 0)) continue;
    const __nv_bfloat16* key =
        slots ? k_hi + ((size_t)bh * hi_stride + s) * kHeadDim
              : static_cast<const __nv_bfloat16*>(a.k.p) + b * a.k.b + h * a.k.h + (s < n ? path[s] : 0) * a.k.t;
    float x[4], sum = 0.f;
    row_values(*reinterpret_cast<const uint2*>(key + 4 * lane), nullptr, lane, x);
    for (int c = slots ? 0 : s; c < n; ++c)
      for (int j = h * G; j < (h + 1) * G; ++j) {
        const __nv_bfloat16* query = static_cast<const __nv_bfloat16*>(a.q.p) + b * a.q.b + j * a.q.h + path[c] * a.q.t;
        const float lse = a.lse[((size_t)b * Hq + j) * a.nodes + path[c]];
        float y[4];
        row_values(*reinterpret_cast<const uint2*>(query + 4 * lane), nullptr, lane, y);
        float d = x[0] * y[0] + x[1] * y[1] + x[2] * y[2] + x[3] * y[3];
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) d += __shfl_xor_sync(0xffffffffu, d, off);
        if (!isinf(lse)) sum += expf(d * a.sm_scale - lse);
      }
    if (lane == 0) {
      if (slots)
        acc[(size_t)bh * hi_stride + s] += sum;
      else
        a.gained[(size_t)bh * a.steps + s] = sum;
    }
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
// (places: the slots, then the path's nodes); a warp to a row quantizes them; then the tokens that stay are written.
constexpr int kCommitThreads = 256;
template <int BITS, int GROUP>
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const CommitArrays c, const PathArgs a) {
  __shared__ int path[kTreeNodes], count, victim[kTreeNodes], place[kTreeNodes];
  __shared__ unsigned long long s_key[kCommitThreads / 32];
  __shared__ int s_at[kCommitThreads / 32];
  const int bh = blockIdx.x, b = bh / c.Hkv, h = bh - b * c.Hkv, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const Commit m = commit_of(a, b, accepted(a.path + (size_t)b * a.steps, a.steps, a.nodes, path, &count), BITS, c.lo_cap);
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
  unsigned long long last_key = 0ull;  // the least entry found so far
  int last_at = -1;
  for (int j = 0; j < m.gone; ++j) {
    unsigned long long best = ~0ull;
    int at = entries;
    for (int e = tid; e < entries; e += kCommitThreads) {
      if (e == free_slot) continue;
      const unsigned long long k = key_of(e);
      const bool left = j == 0 || k > last_key || (k == last_key && e > last_at);
      if (left && (at == entries || k < best)) best = k, at = e;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      const unsigned long long k = __shfl_xor_sync(0xffffffffu, best, off);
      const int e = __shfl_xor_sync(0xffffffffu, at, off);
      if (k < best || (k == best && e < at)) best = k, at = e;
    }
    if (lane == 0) s_key[warp] = best, s_at[warp] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kCommitThreads / 32; ++w)
        if (s_key[w] < s_key[0] || (s_key[w] == s_key[0] && s_at[w] < s_at[0])) s_key[0] = s_key[w], s_at[0] = s_at[w];
      victim[j] = s_at[0];
    }
    __syncthreads();
    last_key = s_key[0], last_at = victim[j];
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

// The lengths after a commit, in a launch of its own: they may be written over those that the commit read.
__global__ void __launch_bounds__(kTreeNodes) commit_lengths_kernel(const PathArgs a, int bits, int lo_cap) {
  __shared__ int path[kTreeNodes], count;
  const int b = blockIdx.x;
  const Commit m = commit_of(a, b, accepted(a.path + (size_t)b * a.steps, a.steps, a.nodes, path, &count), bits, lo_cap);
  if (threadIdx.x) return;
  const int count_in = m.fits ? m.count : 0, gone = m.fits ? m.gone : 0;
  if (a.n_hi_out) a.n_hi_out[b] = m.n_hi + count_in - gone;
  if (a.n_lo_out) a.n_lo_out[b] = m.n_lo + (bits ? gone : 0);
  if (a.next) a.next[b] = a.first[b] + count_in;
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
constexpr int kCopyArrays = 16, kCopyPairs = 256, kCopyThreads = 256, kCopyChunk = 64 * 1024;
struct CopyArgs {
  CopyArray x[kCopyArrays];
  int2 pair[kCopyPairs];
  CopyLengths len;
  int arrays, heads, hi_cap, kch;
};

// Block (pair, chunk, head): its chunk of the bytes that the request keeps of this head, array after array. Pairs run
// fastest, so that those of one source read it from L2.
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyArgs a) {
  const int2 pair = a.pair[blockIdx.x];
  const int h = blockIdx.z;
  const int n_hi = a.len.n_hi ? max(0, min(a.len.n_hi[pair.x], a.hi_cap)) : a.hi_cap;
  const int n_lo = a.len.n_lo ? max(0, min(a.len.n_lo[pair.x], a.len.n_lo_max)) : a.len.n_lo_max;
  if (blockIdx.y == 0 && threadIdx.x == 0) {
    if (a.len.to_slots) a.len.to_slots[pair.y * a.heads + h] = a.len.slots ? a.len.slots[pair.x * a.heads + h] : -1;
    if (h == 0 && a.len.to_n_hi) a.len.to_n_hi[pair.y] = n_hi;
    if (h == 0 && a.len.to_n_lo) a.len.to_n_lo[pair.y] = n_lo;
  }
  const int kept = a.kch ? n_lo / kKchGroup * kKchGroup : n_lo;
  for (int chunk = blockIdx.y;; chunk += gridDim.y) {
    long long begin = (long long)chunk * kCopyChunk, end = begin + kCopyChunk;
    for (int i = 0; i < a.arrays && end > 0; ++i) {
      const CopyArray& x = a.x[i];
      const int rows = x.kind == kHiRows ? n_hi : x.kind == kLoRows ? kept : x.kind == kGroups ? kept / kKchGroup : n_lo - kept;
      const long long bytes = (long long)rows * x.row_bytes;
      const long long lo = max(begin, 0ll), hi = min(end, bytes);
      const char* from = x.from + (((size_t)pair.x * a.heads + h) * x.from_cap + x.from_row) * x.row_bytes;
      char* to = x.to + (((size_t)pair.y * a.heads + h) * x.to_cap + x.to_row) * x.row_bytes;
      for (long long at = lo + 4 * threadIdx.x; at < hi; at += 4 * kCopyThreads)
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
  const dim3 grid((s.hi_cap + kSlots - 1) / kSlots + 1, s.batch * s.heads_kv);
  importance_kernel<<<grid, 256, 0, st>>>(a.cache->acc, static_cast<const __nv_bfloat16*>(a.cache->k_hi), a, s.heads_q,
                                          s.heads_kv, s.hi_stride);
  return cudaGetLastError();
}

cudaError_t launch_commit(const mikv_shape& s, const PathArgs& a, cudaStream_t st) {
  const mikv_cache& k = *a.cache;
  const CommitArrays c = {static_cast<__nv_bfloat16*>(k.k_hi), static_cast<__nv_bfloat16*>(k.v_hi), k.hi_tok, k.acc,
                          static_cast<uint8_t*>(k.k_codes), static_cast<uint8_t*>(k.v_codes),
                          static_cast<__half2*>(k.k_params), static_cast<__half2*>(k.v_params), k.lo_tok, k.balancer,
                          s.heads_kv, s.hi_stride, s.lo_cap};
  void (*kernel)(const CommitArrays, const PathArgs) = nullptr;
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
  kernel<<<s.batch * s.heads_kv, kCommitThreads, 0, st>>>(c, a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || (!a.n_hi_out && !a.n_lo_out && !a.next)) return e;
  commit_lengths_kernel<<<s.batch, kTreeNodes, 0, st>>>(a, s.bits, s.lo_cap);
  return cudaGetLastError();
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
  const int chunks = (int)std::min(std::max(1ll, (most + kCopyChunk - 1) / kCopyChunk), 65535ll);
  for (int first = 0; first < n; first += kCopyPairs) {
    const int count = std::min(kCopyPairs, n - first);
    for (int i = 0; i < count; ++i) a.pair[i] = make_int2(pairs[2 * (first + i)], pairs[2 * (first + i) + 1]);
    copy_kernel<<<dim3(count, chunks, s.heads_kv), kCopyThreads, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace mikv
