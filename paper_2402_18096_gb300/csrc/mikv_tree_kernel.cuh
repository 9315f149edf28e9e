// mikv_tree_kernel.cuh — attention of drafted tokens over the mixed-precision cache on the fifth-generation tensor cores
// (sm_103a). mikv_tree_b2.cu, mikv_tree_b3.cu and mikv_tree_b4.cu instantiate the kernel for one code width each;
// mikv_tree.cu holds the launch and the merge of split parts.
//
// Problem. The N drafted tokens of a request, times the G query heads of a KV head, are R = N G query rows over the same
// keys: the nodes of the tree (one tile of 128, each row sees its ancestors), the important slots (bf16) and the retained
// rows (codes). Row R = node * G + head; 128 rows are a tile (TMEM lanes), two tiles share their keys (PAIR).
//
// Work. An item is a row tile (pair) of one KV head; its key tiles of 128 are the nodes, then the slots, then the retained
// rows. All items' tiles are laid end to end, weighted by what they cost, and every CTA takes an equal run of them; an
// item that lies in several runs is merged by a second kernel. The runs follow from the requests' lengths, which lie in
// device memory, by the same arithmetic in both kernels.
//
// A CTA has two streams, each with a score tile S and an output tile O (128 x 128 fp32) in TMEM: PAIR one row tile each,
// over the same key tiles; otherwise the same rows over alternating key tiles, joined at the end. Roles:
//   warps 0-3, 4-7  the streams' softmax (thread = row = TMEM lane); they also stage the rows' queries
//   warps 8-15      keys and values: packed codes to fp16 tiles in shared memory; bf16 tiles are looked through where
//                   slots or nodes hold nothing (their values may be any bits, and 0 * NaN would reach O)
//   warp 16         copies bf16 tiles (TMA) and asks for codes ahead (L2)
//   warp 17         issues the MMAs: S = Q K^T, O += P V (P over S in TMEM)
//   warp 18         works out the coming items
// All tiles pass one ring of shared memory in the order of their use.
//
// Bound by the chain of a key tile, about 2400 clocks with up to 64 rows: its codes to a tile of keys and one of values
// (1450 each, eight warps), 16 MMAs (87 clocks each, most of them the operands' way out of shared memory) and the hand-overs
// between the roles. 32 requests of up to 32768 tokens, 8 KV heads, 64 rows: 638 us (2.4 TB/s of codes); 4 requests of
// 16384, 508 rows: 174 us (0.78 PFLOP/s).
//
// Precision. A retained key enters as alpha code / b + beta / b, rounded to fp16, so that the query enters as it is: its
// bf16 elements are exact in fp16 once a power of two brings the row's largest to 2^14. (A query divided by the balancer
// and rounded would be off alike for all keys, 1e-5 of lse; roundings of the keys average out.) Requests with few
// retained rows have nothing to average over: there the key's rounding error follows as a second tile (kFineRows).
// Weights are 2^(x - r) with a reference r per row, as in mikv_flash.cuh, in fp16's range for both kinds of tiles.
#pragma once

#include "mikv_flash.cuh"
#include "mikv_tree.h"

namespace mikv {

struct TreeKernelArgs {
  CUtensorMap map_k_hi, map_v_hi;  // bf16 [batch * heads * hi_stride][128], box 64 channels x 128 rows, 128B swizzle
  CUtensorMap map_k, map_v;        // bf16 [batch][heads][nodes][128], box 64 channels x 128 nodes
  TreeArgs a;
  int rows, m_blocks, log2_G;      // rows of a KV head; row tiles (pairs)
  int twin;                        // the rows of a tile (up to 64) stand in it twice
  uint32_t* prefix;                // [batch + 1] costs of all items before each request (for the merge)
  float* part_o;                   // [2 * CTAs][rows of an item][128]
  float* part_lse;                 // [2 * CTAs][rows of an item], log2
};

template <int BITS>
cudaError_t launch_tree_kernel(const TreeKernelArgs& p, bool pair, int grid, cudaStream_t st);

namespace tree {

using flash::kHalfBytes;
using flash::kLn2;
using flash::kLog2e;
using flash::kTile;
using flash::kTileBytes;

constexpr int kSoftThreads = 256, kCodeThreads = 256, kThreads = 640;
constexpr int kCodeWarp = 8, kCopyWarp = 16, kMmaWarp = 17, kPlanWarp = 18;
constexpr int kItemRing = 4, kItemReaders = 18, kBadRing = 8;
constexpr int kTmemCols = 512;  // S0, S1, O0, O1
constexpr int kExPitch = 33;    // floats of a row's 32 channels in the exchange (padded against conflicts)

// Costs of tiles, for the runs: the nodes (with the start and the end of an item), slots, retained rows, those of few
// (kFineRows). With 2, 2, 1, 1 the same calls took 690 us in place of 642 (32 requests of up to 32768 tokens, 64 rows), 203 of
// 173 (4 of 16384, 508 rows) and 104 of 85 (8 of 118 .. 4096 retained rows, 33 rows).
constexpr int kCostNodes = 3, kCostHi = 1, kCostLo = 1, kCostFine = 2;
constexpr int kLeastRun = 3;       // cost of a run at least (6: 29.7 us where 1, 3 and 4 take 23.4, 32 items of 2047 tokens)
constexpr int kFineRows = 1024;    // requests with up to this many retained rows have their keys in two tiles
constexpr int kAhead = 6;          // tiles of codes asked for ahead (L2)

template <bool PAIR_>
struct Layout {
  static constexpr bool PAIR = PAIR_;
  static constexpr int kItemRows = PAIR ? 2 * kTile : kTile;
  static constexpr int kQ = PAIR ? 4 : 2;       // query tiles: per row tile one in bf16 and one in fp16
  static constexpr int kStages = PAIR ? 3 : 4;  // tiles in the ring
  // Loads of an item: the first kLead K tiles, then V tile u and K tile u + kLead for u = 0, 1, ...
  static constexpr int kLead = PAIR ? 1 : 2;
  static constexpr int kBars = 3 * kStages + 10 + 2 + 2 * kItemRing + 1;
  static constexpr int kParts = PAIR ? 0 : 4 * kTile * 4, kExchange = PAIR ? 0 : 2 * (kTile / 2) * kExPitch * 4;
  static constexpr int kTables = 8 * kBars + 8 + 2 * kHeadDim * 4 + kParts + kExchange;
  static constexpr int kSmem = 1024 + (kQ + kStages) * kTileBytes + kTables;
  static_assert(kSmem <= 227 * 1024 - 512, "shared memory of one CTA");
  uint32_t base;
  __device__ uint32_t q(int m, bool f16) const { return base + (2 * m + (f16 ? 1 : 0)) * kTileBytes; }
  __device__ uint32_t stage(int s) const { return base + (kQ + s) * kTileBytes; }
  __device__ uint32_t bar(int i) const { return base + (kQ + kStages) * kTileBytes + 8 * i; }
  // 1 / balancer of an item's channels: in fp32 or, of 8 channels each, the fp16 nearest to it and to what that leaves
  __device__ uint32_t inverse(int round) const { return base + (kQ + kStages) * kTileBytes + (8 * kBars + 15) / 16 * 16 + (round & 1) * kHeadDim * 4; }
  __device__ uint32_t parts() const { return inverse(0) + 2 * kHeadDim * 4; }
  __device__ uint32_t exchange(int w) const { return parts() + kParts + w * (kTile / 2) * kExPitch * 4; }
  __device__ uint32_t full(int s) const { return bar(s); }                  // a bf16 tile landed; a code tile may be written
  __device__ uint32_t ready(int s) const { return bar(kStages + s); }       // a tile may be multiplied
  __device__ uint32_t empty(int s) const { return bar(2 * kStages + s); }   // it is not needed any more
  __device__ uint32_t sfull(int w) const { return bar(3 * kStages + w); }   // scores of stream w
  // of half a tile (64 keys): weights written (and O rescaled for them); O += P V done
  __device__ uint32_t pready(int w, int half) const { return bar(3 * kStages + 2 + 2 * w + half); }
  __device__ uint32_t odone(int w, int half) const { return bar(3 * kStages + 6 + 2 * w + half); }
  __device__ uint32_t qfull() const { return bar(3 * kStages + 10); }       // an item's queries are staged
  __device__ uint32_t qfree() const { return bar(3 * kStages + 11); }       // its last scores have read them
  __device__ uint32_t itemfull(int i) const { return bar(3 * kStages + 12 + i % kItemRing); }
  __device__ uint32_t itemfree(int i) const { return bar(3 * kStages + 12 + kItemRing + i % kItemRing); }
  __device__ uint32_t drain() const { return bar(kBars - 1); }
  __device__ static constexpr int arrivals(int i) {
    if (i >= kStages && i < 2 * kStages) return kCodeThreads / 32;
    if (i >= 3 * kStages + 2 && i < 3 * kStages + 6) return 4;  // the softmax warps of the stream
    if (i == 3 * kStages + 10) return kSoftThreads / 32;
    if (i >= 3 * kStages + 12 + kItemRing && i < kBars - 1) return kItemReaders;
    return 1;
  }
};

// The key tiles of a request's items, and the costs before each.
struct Tiles {
  int hi, lo, each;  // tiles of slots, of retained rows; cost of one of the latter
  __device__ Tiles(const HeldArgs& held, int b) : hi((held.hi(b) + kTile - 1) / kTile) {
    const int rows = held.lo(b);
    lo = (rows + kTile - 1) / kTile, each = rows <= kFineRows ? kCostFine : kCostLo;
  }
  __device__ int count() const { return 1 + hi + lo; }
  __device__ int cost() const { return kCostNodes + kCostHi * hi + each * lo; }
  __device__ int before(int t) const {
    return t == 0 ? 0 : kCostNodes + (t <= hi ? kCostHi * (t - 1) : kCostHi * hi + each * (t - 1 - hi));
  }
  // the first tile that begins at x or later
  __device__ int first(int x) const {
    if (x <= 0) return 0;
    x -= kCostNodes;
    const int t = x <= 0 ? 0 : x <= kCostHi * hi ? (x + kCostHi - 1) / kCostHi : hi + (x - kCostHi * hi + each - 1) / each;
    return min(t + 1, count());
  }
};

// CTA (or warp) c has the costs [first(c), first(c + 1)) of all: shares that differ by one at most. In 32 bits (sizes that
// could pass them are refused, tree_sizes_ok), for 64-bit divisions are long and a small call runs its code once, cold.
struct Runs {
  uint32_t share, more;  // the first `more` runs have one more
  int n;
  __device__ Runs(uint32_t total, int ctas, int least = kLeastRun) : n((int)max(1u, min((uint32_t)ctas, total / least))) {
    share = total / n, more = total - share * n;
  }
  __device__ uint32_t first(int c) const { return share * c + min((uint32_t)c, more); }
  __device__ int owner(uint32_t x) const {
    const uint32_t larger = (share + 1) * more;
    const bool in = x < larger;
    return (in ? 0 : more) + (in ? x : x - larger) / (in ? share + 1 : max(1u, share));
  }
};

struct alignas(16) ItemData {
  int b, h, m_block, slot;  // slot: where the item's part goes, -1: the whole item is here
  int t0, t1, hi_tiles, n_hi;
  int n_lo, free_slot, fine, valid;
  __device__ int n() const { return t1 - t0; }
  __device__ bool codes(int t) const { return t > hi_tiles; }
};

// Barrier of a role's warps that tells all of them whether one of them has failed.
template <int ID, int THREADS>
__device__ __forceinline__ bool group_sync(bool failed) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)failed), "n"(ID), "n"(THREADS)
      : "memory");
  return any != 0;
}

__device__ __forceinline__ void sts128(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w));
}
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t x) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(x) : "memory");
}
__device__ __forceinline__ void sts16(uint32_t addr, uint16_t x) {
  asm volatile("st.shared.b16 [%0], %1;" ::"r"(addr), "h"(x) : "memory");
}
// Asks for `bytes` at p (both multiples of 16) to be brought into L2.
__device__ __forceinline__ void prefetch_l2_bulk(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// S (128 x 128) = (or +=) query tile x key tile^T.
__device__ __forceinline__ void mma_keys(uint32_t d, uint32_t q, uint32_t k, bool f16, bool accumulate) {
  const uint32_t idesc = f16 ? umma_idesc_16(true, kTile, kTile, false) : umma_idesc_16(false, kTile, kTile, false);
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    const uint32_t off = (ks >> 2) * kHalfBytes + (ks & 3) * 32;
    umma_bf16(d, umma_desc_sw128(q + off), umma_desc_sw128(k + off), idesc, ks > 0 || accumulate ? 1u : 0u);
  }
}
// O (128 x 128) += P (TMEM) x value tile, 64 of the keys.
__device__ __forceinline__ void mma_values(uint32_t d, uint32_t p, uint32_t v, int half, bool f16, bool accumulate) {
  const uint32_t idesc = f16 ? umma_idesc_16(true, kTile, kTile, true) : umma_idesc_16(false, kTile, kTile, true);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int ks = 4 * half + i;
    umma_16_ts(d, p + 8 * ks, umma_desc_rows_sw128(v + ks * 16 * 128, kHalfBytes), idesc, ks > 0 || accumulate ? 1u : 0u);
  }
}

// The packed codes of half a retained row, as a thread takes them: half j holds the channels 16 m + 8 j + 0 .. 7 of every
// m = 0 .. 7, in the 16-byte blocks j (and 2 + j) of the row's plane; and the row's parameters, a pair per 32 channels.
template <int BITS>
struct Codes {
  static constexpr int kWords = BITS == 4 ? 8 : 4;
  uint32_t w[kWords], top[BITS == 3 ? 4 : 1], pair[4];
  // codes, params: those of row 0
  __device__ __forceinline__ void load(const uint8_t* codes, const uint32_t* params, uint32_t row, int j, int group) {
    auto get = [](const void* p) { return __ldg(static_cast<const uint4*>(p)); };
    const uint8_t* at = codes + (uint64_t)row * (16 * BITS);
    const uint4 x = get(at + 16 * j);
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    if constexpr (BITS == 4) {
      const uint4 y = get(at + 16 * j + 32);
      w[4] = y.x, w[5] = y.y, w[6] = y.z, w[7] = y.w;
    }
    if constexpr (BITS == 3) {
      const uint4 y = get(at + 32);
      top[0] = y.x, top[1] = y.y, top[2] = y.z, top[3] = y.w;
    }
    if (group == 32) {
      const uint4 y = get(params + 4 * (uint64_t)row);
      pair[0] = y.x, pair[1] = y.y, pair[2] = y.z, pair[3] = y.w;
    } else if (group == 64) {
      const uint2 y = __ldg(reinterpret_cast<const uint2*>(params + 2 * (uint64_t)row));
      pair[0] = pair[1] = y.x, pair[2] = pair[3] = y.y;
    } else {
      pair[0] = pair[1] = pair[2] = pair[3] = __ldg(params + row);
    }
  }
  // The same codes (channels 16 m + 8 j + 2 q and the next) as Fields gives them, for any m at run time.
  __device__ __forceinline__ __half2 code(int m, int q, int j) const {
    uint32_t x;
    if constexpr (BITS == 4) {
      x = and_or((m < 4 ? w[q] : w[4 + q]) >> (4 * (m & 3)), 0x000F000Fu, 0x64006400u);
    } else {
      x = and_or(w[q] >> (2 * m), 0x00030003u, 0x64006400u);
      if constexpr (BITS == 3) x |= ((top[q] >> (2 * m + j)) & 0x00010001u) << 2;
    }
    return __hsub2(u32_as_h2(x), u32_as_h2(0x64006400u));
  }
};

// The codes of channels 16 m + 8 j + 2 q and the next of a row, as exact fp16 numbers: the field's bits stay where they are
// (bit s of each 16-bit unit, after one shift of the word for the upper fields) under the exponent that makes bit s count
// 1, which is then taken off.
template <int BITS>
struct Fields {
  static constexpr int kShift = BITS == 2 ? 10 : 8, kUpper = BITS == 2 ? 5 : BITS == 3 ? 4 : 2;  // from field kUpper on
  uint32_t lo[BITS == 4 ? 8 : 4], up[BITS == 4 ? 8 : 4], lo_top[BITS == 3 ? 4 : 1], up_top[BITS == 3 ? 4 : 1];
  __device__ __forceinline__ Fields(const Codes<BITS>& c, int j) {
#pragma unroll
    for (int i = 0; i < Codes<BITS>::kWords; ++i) lo[i] = c.w[i], up[i] = c.w[i] >> kShift;
    if constexpr (BITS == 3) {
#pragma unroll
      for (int i = 0; i < 4; ++i) lo_top[i] = (c.top[i] >> j) << 2, up_top[i] = (c.top[i] >> j) >> 6;
    }
  }
  __device__ __forceinline__ __half2 code(int m, int q) const {
    const int f = BITS == 4 ? m & 3 : m, width = BITS == 4 ? 4 : 2;
    const bool upper = f >= kUpper;
    const int s = width * f - (upper ? kShift : 0);
    const uint32_t magic = 0x64006400u - 0x04000400u * s, mask = BITS == 4 ? 0x000F000Fu : 0x00030003u;
    const int i = BITS == 4 ? 4 * (m >> 2) + q : q;
    uint32_t x = and_or(upper ? up[i] : lo[i], mask << s, magic);
    if constexpr (BITS == 3) x = and_or(upper ? up_top[q] : lo_top[q], 0x00040004u << s, x);
    return __hsub2(u32_as_h2(x), u32_as_h2(magic));
  }
};

// Where chunk `c` (8 channels) of a key lies in a tile.
__device__ __forceinline__ uint32_t chunk_at(uint32_t tile, int key, int c) {
  return tile + (c >> 3) * kHalfBytes + key * 128 + (((c & 7) ^ (key & 7)) << 4);
}

template <int BITS, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) tree_kernel(const __grid_constant__ TreeKernelArgs p) {
  using L = Layout<PAIR>;
  const TreeArgs& a = p.a;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;
  __shared__ ItemData s_item[kItemRing];
  __shared__ uint32_t s_bad[kBadRing][4];  // nodes whose value holds an infinity or NaN
  volatile int* fail = &s_fail;
  L sm;
  sm.base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

  if (tid < L::kBars) mbar_init(sm.bar(tid), L::arrivals(tid));
  if (tid == 0) s_fail = 0;
  fence_mbar_init();
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&s_tmem), kTmemCols);
  if (tid == 32 * kCopyWarp) {
    prefetch_tensormap(&p.map_k_hi);
    prefetch_tensormap(&p.map_v_hi);
    prefetch_tensormap(&p.map_k);
    prefetch_tensormap(&p.map_v);
  }
  tcgen05_before_sync();
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);
  grid_dependency_wait();
  allow_dependent_launch();  // (the merge)

  // The description of the item of a round (uniform); false when a wait gave up.
  auto next_item = [&](int round, ItemData& x) {
    const bool ok = mbar_wait_warp(sm.itemfull(round), (round / kItemRing) & 1, fail);
    const int* d = reinterpret_cast<const int*>(&s_item[round % kItemRing]);
    int* to = reinterpret_cast<int*>(&x);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(ItemData) / 4); ++i) to[i] = __shfl_sync(0xffffffffu, d[i], 0);
    __syncwarp();
    if (lane == 0) mbar_arrive(sm.itemfree(round));
    return ok;
  };
  // Registers go to the softmax warps: 256 x 128 + 256 x 88 + 128 x 48 = 640 x 96.
  if (warp >= kCopyWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == kCopyWarp) {
      int c = 0;  // loads so far
      int last[L::kStages];  // the last copy into each stage
#pragma unroll
      for (int s = 0; s < L::kStages; ++s) last[s] = -1;
      bool ok = true;
      ItemData x = {};
      for (int round = 0; ok; ++round) {
        ok = next_item(round, x);
        if (!ok || !x.valid) break;
        if (lane == 0) {
          const int bh = x.b * a.heads_kv + x.h;
          const int row_bytes = 4 * (kHeadDim / a.group);
          auto ask = [&](int t, bool values) {  // the codes and parameters of tile t into L2
            const int r = (t - 1 - x.hi_tiles) * kTile, rows = min(kTile, x.n_lo - r);
            if (t >= x.t1 || rows <= 0) return;
            const size_t row = (size_t)bh * a.lo_cap + r;
            prefetch_l2_bulk((values ? a.v_codes : a.k_codes) + row * 16 * BITS, rows * 16 * BITS);
            prefetch_l2_bulk(reinterpret_cast<const char*>(values ? a.v_params : a.k_params) + row * row_bytes,
                             (rows * row_bytes + 15) & ~15);
          };
          int asked = max(x.t0, 1 + x.hi_tiles);  // tiles asked for, two at a time
          const int n = x.n();
          // V tile u, then K tile u + kLead. Every stage passes through here in its turn, those that the code warps write
          // too: a role that waited for some phases of a barrier only could take another of the same parity for its own.
#pragma unroll 1
          for (int i = -2 * L::kLead; ok && i < 2 * n; ++i) {
            const bool values = !(i & 1);
            const int u = (i >> 1) + (values ? 0 : L::kLead), t = x.t0 + u;
            if (values ? i < 0 : u >= n) continue;
            const bool code = x.codes(t);
            for (int part = code && x.fine && !values ? 2 : 1; ok && part > 0; --part) {
              const int s = c % L::kStages;
              ok = c < L::kStages || mbar_wait_role(sm.empty(s), ((c / L::kStages) & 1) ^ 1, fail);
              if (!ok) break;
              if (code) {
                mbar_arrive(sm.full(s));
#pragma unroll
                for (int q = 0; q < L::kStages; ++q)
                  if (q == s) last[q] = -1;  // (what was copied here has been multiplied)
              } else {
                mbar_arrive_expect_tx(sm.full(s), kTileBytes);
                const CUtensorMap* map = t == 0 ? (values ? &p.map_v : &p.map_k) : (values ? &p.map_v_hi : &p.map_k_hi);
                const int row = bh * a.hi_stride + (t - 1) * kTile;
#pragma unroll
                for (int ch = 0; ch < kHeadDim; ch += 64) {
                  const uint32_t to = sm.stage(s) + (ch ? kHalfBytes : 0);
                  if (t == 0)
                    tma_load_4d(to, map, ch, 0, x.h, x.b, sm.full(s));
                  else
                    tma_load_2d(to, map, ch, row, sm.full(s));
                }
#pragma unroll
                for (int q = 0; q < L::kStages; ++q)
                  if (q == s) last[q] = c;
              }
              ++c;
            }
            for (int k = 0; k < 2 && asked < min(x.t1, t + 1 + kAhead); ++k, ++asked) {
              ask(asked, false);
              ask(asked, true);
            }
          }
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
      }
      if (lane == 0) {  // no copy may outlive the CTA, whatever became of the other roles
#pragma unroll
        for (int s = 0; s < L::kStages; ++s)
          if (last[s] >= 0 && !mbar_wait(sm.full(s), (last[s] / L::kStages) & 1)) record_error(a.status, kErrDrainTimeout);
      }
      __syncwarp();
    } else if (warp == kMmaWarp) {  // the whole warp, converged; one lane issues
      const bool leader = elect_one();
      int c = 0;
      int tiles[2] = {0, 0};  // tiles of each stream whose weights were consumed
      auto commit = [&](uint32_t bar) {
        if (leader) umma_commit(bar);
      };
      auto wait_ready = [&](int load) {
        const bool ok = mbar_wait_warp(sm.ready(load % L::kStages), (load / L::kStages) & 1, fail);
        tcgen05_after_sync();
        return ok;
      };
      auto release = [&](int load) { commit(sm.empty(load % L::kStages)); };
      // scores of stream w from one key tile (and the second one, of the roundings)
      auto scores = [&](int w, int load, bool f16, bool fine) {
        if (leader) {
          const uint32_t q = sm.q(PAIR ? w : 0, f16);
          mma_keys(tmem + 128 * w, q, sm.stage(load % L::kStages), f16, false);
          if (fine) mma_keys(tmem + 128 * w, q, sm.stage((load + 1) % L::kStages), f16, true);
          umma_commit(sm.sfull(w));
        }
      };
      auto values = [&](int w, int load, bool f16, bool first) {
        const uint32_t v = sm.stage(load % L::kStages);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!mbar_wait_warp(sm.pready(w, half), (w ? tiles[1] : tiles[0]) & 1, fail)) return false;
          tcgen05_after_sync();
          if (leader) {
            mma_values(tmem + 256 + 128 * w, tmem + 128 * w, v, half, f16, !first);
            umma_commit(sm.odone(w, half));
          }
        }
        (w ? tiles[1] : tiles[0]) += 1;
        return true;
      };
      bool ok = true;
      ItemData x = {};
      for (int round = 0; ok; ++round) {
        ok = next_item(round, x);
        if (!ok || !x.valid) break;
        const int n = x.n();
        ok = mbar_wait_warp(sm.qfull(), round & 1, fail);
        tcgen05_after_sync();
        // keys of tile t (both streams where PAIR, else stream w): waited for, multiplied, released
        auto keys_ready = [&](int t) {
          const bool fine = x.fine && x.codes(t);
          return wait_ready(c) && (!fine || wait_ready(c + 1));
        };
        auto keys_done = [&](int t, int& load) {
          const bool fine = x.fine && x.codes(t);
          release(load);
          if (fine) release(load + 1);
          load += fine ? 2 : 1;
        };
        auto is_fine = [&](int t) { return x.fine && x.codes(t); };
        if constexpr (PAIR) {
          ok = ok && keys_ready(x.t0);
          if (ok) {
#pragma unroll
            for (int w = 0; w < 2; ++w) scores(w, c, x.codes(x.t0), is_fine(x.t0));
            keys_done(x.t0, c);
            if (n == 1) commit(sm.qfree());
          }
#pragma unroll 1
          for (int u = 0; ok && u < n; ++u) {
            const int t = x.t0 + u, cv = c;
            ok = wait_ready(cv);
            ++c;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              if (ok) ok = values(w, cv, x.codes(t), u == 0);
              if (ok && u + 1 < n) {
                if (w == 0) ok = keys_ready(t + 1);
                if (ok) scores(w, c, x.codes(t + 1), is_fine(t + 1));
              }
            }
            if (ok) {
              release(cv);
              if (u + 1 < n) keys_done(t + 1, c);
              if (u + 2 == n) commit(sm.qfree());
            }
          }
        } else {  // step u: the product of tile u (from 0 on), then the scores of tile u + 2; streams in turn
#pragma unroll 1
          for (int u = -2; ok && u < n; ++u) {
            const int w = u & 1, t = x.t0 + u;
            if (u >= 0) {
              ok = wait_ready(c) && values(w, c, x.codes(t), u < 2);
              if (ok) {
                release(c);
                ++c;
              }
            }
            if (ok && u + 2 < n) {
              ok = keys_ready(t + 2);
              if (ok) {
                scores(w, c, x.codes(t + 2), is_fine(t + 2));
                keys_done(t + 2, c);
                if (u + 3 == n) commit(sm.qfree());
              }
            }
          }
        }
      }
      commit(sm.drain());  // every MMA issued has completed once this arrives
      if (!mbar_wait(sm.drain(), 0) && lane == 0) record_error(a.status, kErrDrainTimeout);
      __syncwarp();
    } else if (warp == kPlanWarp) {  // the coming items, up to kItemRing ahead, and the end
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
      const int per_set = a.heads_kv * p.m_blocks;
      // costs of the items of requests b0 .. b0 + lane, and of this lane's
      auto scan = [&](int b0, uint32_t& mine) {
        mine = b0 + lane < a.batch ? Tiles(a.held, b0 + lane).cost() * per_set : 0;
        uint32_t sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(0xffffffffu, sum, o);
          if (lane >= o) sum += y;
        }
        return sum;
      };
      uint32_t all = 0, mine;
#pragma unroll 1
      for (int b0 = 0; b0 < a.batch; b0 += 32) {
        const uint32_t sum = scan(b0, mine);
        if (blockIdx.x == 0 && b0 + lane < a.batch) p.prefix[b0 + lane] = all + sum - mine;
        all += __shfl_sync(0xffffffffu, sum, 31);
      }
      if (blockIdx.x == 0 && lane == 0) p.prefix[a.batch] = all;
      const Runs runs(all, gridDim.x);
      uint32_t from = 0, to = 0, start = 0;  // this CTA's run; costs before the item at hand
      if ((int)blockIdx.x < runs.n) from = runs.first(blockIdx.x), to = runs.first(blockIdx.x + 1);
      int b = 0, in_set = 0;
#pragma unroll 1
      for (int b0 = 0; from < to && b0 < a.batch; b0 += 32) {
        const uint32_t sum = scan(b0, mine), total = __shfl_sync(0xffffffffu, sum, 31);
        if (from < start + total) {
          const int at = __ffs(__ballot_sync(0xffffffffu, start + sum > from)) - 1;
          b = b0 + at;
          start += __shfl_sync(0xffffffffu, sum - mine, at);
          const uint32_t cost = Tiles(a.held, b).cost();
          in_set = (int)((from - start) / cost);
          start += in_set * cost;
          break;
        }
        start += total;
      }
      bool ok = true;
#pragma unroll 1
      while (ok && start < to) {
        const Tiles tl(a.held, b);
        ItemData x = {};
        x.b = b;
        x.h = in_set / p.m_blocks;
        x.m_block = in_set - x.h * p.m_blocks;
        x.hi_tiles = tl.hi;
        x.n_hi = a.held.hi(b);
        x.n_lo = a.held.lo(b);
        x.free_slot = a.held.free_slot(b * a.heads_kv + x.h, x.n_hi);
        x.fine = x.n_lo <= kFineRows;
        x.t0 = tl.first((int)(from - start));
        x.t1 = tl.first((int)(to - start));
        x.slot = x.t0 == 0 && x.t1 == tl.count() ? -1 : 2 * (int)blockIdx.x + (x.t0 == 0);
        x.valid = 1;
        if (x.t0 < x.t1) ok = publish(x);
        start += tl.cost();
        if (++in_set == per_set) in_set = 0, ++b;
      }
      if (ok) publish(ItemData{});
    }
  } else if (warp >= kCodeWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    // The thread's place in a tile: a key and half of its channels. Eight lanes that store together have keys of one
    // parity, so that their chunks fall on different banks; a warp reads 16 rows as they lie.
    const int w = warp - kCodeWarp, quarter = lane >> 3, j = lane & 1;
    const int key = 16 * w + 8 * (quarter >> 1) + (quarter & 1) + 2 * ((lane & 7) >> 1);
    int c = 0;
    bool ok = true;
    ItemData x = {};
    for (int round = 0;; ++round) {
      if (ok) ok = next_item(round, x);
      bool wide = false;  // a balancer too far from 1 for fp16 arithmetic
      if (ok && x.valid) {
        const int ct = tid - 32 * kCodeWarp;
        if (ct < kHeadDim) {
          const float inv = a.balancer ? 1.f / a.balancer[x.h * kHeadDim + ct] : 1.f;
          wide = !(inv >= 0x1p-4f && inv <= 0x1p10f);
          sts32(sm.inverse(round) + 4 * ct, __float_as_uint(inv));
        }
      }
      if (group_sync<2, kCodeThreads>(!ok) || !x.valid) break;
      const bool exact = group_sync<2, kCodeThreads>(wide) || x.fine;  // keys in fp32 arithmetic
      const uint32_t inverse = sm.inverse(round);
      if (!exact) {  // in place: of chunk c (8 channels) 16 bytes of the fp16 nearest to 1 / b, 16 of what that leaves
        const int ct = tid - 32 * kCodeWarp;
        uint32_t bits = 0;
        if (ct < kHeadDim) {
          const float inv = __uint_as_float(lds32(inverse + 4 * ct));
          const __half h = __float2half_rn(inv);
          bits = h2_as_u32(__halves2half2(h, __float2half_rn(inv - __half2float(h))));
        }
        if (group_sync<2, kCodeThreads>(false)) break;
        if (ct < kHeadDim) {
          sts16(inverse + 32 * (ct >> 3) + 2 * (ct & 7), (uint16_t)bits);
          sts16(inverse + 32 * (ct >> 3) + 16 + 2 * (ct & 7), (uint16_t)(bits >> 16));
        }
        if (group_sync<2, kCodeThreads>(false)) break;
      }
      // Rows past the last one repeat it: their keys are masked, and their weights of 0 need finite values only where the
      // last row's are.
      const size_t row0 = (size_t)(x.b * a.heads_kv + x.h) * a.lo_cap, pair0 = row0 * (kHeadDim / a.group);
      const uint32_t* params[2] = {reinterpret_cast<const uint32_t*>(a.k_params) + pair0,
                                   reinterpret_cast<const uint32_t*>(a.v_params) + pair0};
      const uint8_t* codes[2] = {a.k_codes + row0 * (16 * BITS), a.v_codes + row0 * (16 * BITS)};
      const int first_codes = max(x.t0, 1 + x.hi_tiles);
      // The codes of the next key tile and of the next value tile are on their way while the last ones are worked on.
      Codes<BITS> next_k, next_v;
      auto row_of = [&](int t) { return (uint32_t)min((t - 1 - x.hi_tiles) * kTile + key, x.n_lo - 1); };
      if (first_codes < x.t1) {
        next_k.load(codes[0], params[0], row_of(first_codes), j, a.group);
        next_v.load(codes[1], params[1], row_of(first_codes), j, a.group);
      }
      const int n = x.n();
      auto landed = [&](int load) {  // or, for codes, the stage is free
        return mbar_wait_warp(sm.full(load % L::kStages), (load / L::kStages) & 1, fail);
      };
      auto done = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.ready(c % L::kStages));
        ++c;
      };
      // V tile u, then K tile u + kLead
#pragma unroll 1
      for (int i = -2 * L::kLead; ok && i < 2 * n; ++i) {
        const bool values = !(i & 1);
        const int u = (i >> 1) + (values ? 0 : L::kLead), t = x.t0 + u;
        if (values ? i < 0 : u >= n) continue;
        ok = landed(c);
        if (!ok) break;
        const uint32_t tile = sm.stage(c % L::kStages);
        if (!x.codes(t)) {
          if (values) {  // rows that hold no token may hold any bits
            bool blank, bad = false;
            if (t == 0) {
              const uint4 mw = key < a.nodes ? __ldg(a.masks + (size_t)x.b * a.nodes + key) : make_uint4(0u, 0u, 0u, 0u);
              const uint32_t word = key < 64 ? (key < 32 ? mw.x : mw.y) : (key < 96 ? mw.z : mw.w);
              blank = !(word >> (key & 31) & 1);
#pragma unroll 1
              for (int m = 0; m < 8; ++m) bad |= flash::any_nonfinite<false>(flash::lds128(chunk_at(tile, key, 2 * m + j)));
              bad = bad && !blank;
              bad |= __shfl_xor_sync(0xffffffffu, bad, 1);  // the other half of the channels
              // the warp's keys are 16 w .. 16 w + 15: halves of a word, each written by one warp
              const uint32_t bits = __ballot_sync(0xffffffffu, bad && j == 0);
              uint32_t sorted = 0;
#pragma unroll
              for (int k = 0; k < 16; ++k) {  // the lane of key k (j = 0)
                const int of = 8 * (2 * (k >> 3) + (k & 1)) + 2 * ((k & 7) >> 1);
                sorted |= (bits >> of & 1u) << k;
              }
              if (lane == 0) reinterpret_cast<uint16_t*>(s_bad[round % kBadRing])[w] = (uint16_t)sorted;
            } else {
              const int slot = (t - 1) * kTile + key;
              blank = slot >= x.n_hi || slot == x.free_slot;
            }
            if (blank || bad) {
#pragma unroll 1
              for (int m = 0; m < 8; ++m) flash::sts128_zero(chunk_at(tile, key, 2 * m + j));
              fence_async();
            }
          }
          done();
        } else if (values) {
          const Fields<BITS> f(next_v, j);
#pragma unroll
          for (int m = 0; m < 8; ++m) {
            const __half2 pr = u32_as_h2(next_v.pair[m >> 1]), al = __low2half2(pr), be = __high2half2(pr);
            uint32_t y[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = h2_as_u32(__hfma2(f.code(m, q), al, be));
            sts128(chunk_at(tile, key, 2 * m + j), y[0], y[1], y[2], y[3]);
          }
          fence_async();
          done();
          // (behind the fence and the arrival, which wait for loads under way)
          if (t + 1 < x.t1) next_v.load(codes[1], params[1], row_of(t + 1), j, a.group);
        } else {
          if (!exact) {
            const Fields<BITS> f(next_k, j);
            const uint4* table = reinterpret_cast<const uint4*>(smem_raw + (inverse - smem_u32(smem_raw)));
#pragma unroll
            for (int m = 0; m < 8; ++m) {
              const __half2 pr = u32_as_h2(next_k.pair[m >> 1]), al = __low2half2(pr), be = __high2half2(pr);
              const uint4 n4 = table[2 * (2 * m + j)], r4 = table[2 * (2 * m + j) + 1];
              const uint32_t near[4] = {n4.x, n4.y, n4.z, n4.w}, rest[4] = {r4.x, r4.y, r4.z, r4.w};
              uint32_t y[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const __half2 k = __hfma2(f.code(m, q), al, be);
                y[q] = h2_as_u32(__hfma2(k, u32_as_h2(near[q]), __hmul2(k, u32_as_h2(rest[q]))));
              }
              sts128(chunk_at(tile, key, 2 * m + j), y[0], y[1], y[2], y[3]);
            }
          } else {
            if (x.fine) ok = landed(c + 1);
            if (!ok) break;
            const uint32_t second = sm.stage((c + 1) % L::kStages);
#pragma unroll 1
            for (int m = 0; m < 8; ++m) {
              const float2 pr = __half22float2(u32_as_h2(m < 4 ? (m < 2 ? next_k.pair[0] : next_k.pair[1])
                                                               : (m < 6 ? next_k.pair[2] : next_k.pair[3])));
              uint32_t y[4], z[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const uint32_t at = inverse + 64 * m + 32 * j + 8 * q;
                const float2 cd = __half22float2(next_k.code(m, q, j));
                const float k0 = fmaf(pr.x, cd.x, pr.y) * __uint_as_float(lds32(at));
                const float k1 = fmaf(pr.x, cd.y, pr.y) * __uint_as_float(lds32(at + 4));
                y[q] = pack_f16(k0, k1);
                const float2 h = __half22float2(u32_as_h2(y[q]));
                z[q] = pack_f16(k0 - h.x, k1 - h.y);
              }
              sts128(chunk_at(tile, key, 2 * m + j), y[0], y[1], y[2], y[3]);
              if (x.fine) sts128(chunk_at(second, key, 2 * m + j), z[0], z[1], z[2], z[3]);
            }
          }
          fence_async();
          done();
          if (x.fine) done();
          if (t + 1 < x.t1) next_k.load(codes[0], params[0], row_of(t + 1), j, a.group);
        }
      }
    }
  } else {  // softmax warps
    asm volatile("setmaxnreg.inc.sync.aligned.u32 128;");
    constexpr float kDrop = flash::ref_drop<true>(), kSlack = flash::ref_slack<true>(), kSumMax = flash::sum_max<true>();
    const int stream = warp >> 2, r = tid & (kTile - 1);
    const bool twin = !PAIR && p.twin, upper = twin && (warp & 2);  // upper: the second copy of the rows
    const int row = twin ? r & (kTile / 2 - 1) : r;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t ts = tmem + 128 * stream + lanes, to = tmem + 256 + 128 * stream + lanes;
    const float scale = a.sm_scale * kLog2e;
    float* s_part = reinterpret_cast<float*>(smem_raw + (sm.parts() - smem_u32(smem_raw)));  // [stream][ref, sum][row]
    int tiles = 0;  // tiles done, over all items
    ItemData x = {};
    // The thread's row of an item: its node and head, whether there is one, what it sees of the tree, the scale of its
    // fp16 query.
    int node = 0, head = 0;
    bool real = false;
    uint32_t mask[4];
    float scale16 = 0.f;
    // Stages the queries of an item (PAIR: both forms of the stream's row tile; else stream 0 bf16 and stream 1 fp16).
    auto stage_rows = [&](int round) {
      const int R = (PAIR ? 2 * x.m_block + stream : x.m_block) * kTile + row;
      node = R >> p.log2_G;
      head = x.h * a.G + (R & (a.G - 1));
      real = false;
      mask[0] = mask[1] = mask[2] = mask[3] = 0u;
      if (R < p.rows) {
        const uint4 mw = __ldg(a.masks + (size_t)x.b * a.nodes + node);
        mask[0] = mw.x, mask[1] = mw.y, mask[2] = mw.z, mask[3] = mw.w;
        const uint32_t word = node < 64 ? (node < 32 ? mw.x : mw.y) : (node < 96 ? mw.z : mw.w);
        real = word >> (node & 31) & 1;
      }
      const uint4* q = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q.p) + x.b * a.q.b + head * a.q.h +
                                                      node * a.q.t);
      auto low = [](uint32_t v) { return __uint_as_float(v << 16); };
      auto high = [](uint32_t v) { return __uint_as_float(v & 0xffff0000u); };
      auto chunk = [&](int i) { return real ? __ldg(q + i) : make_uint4(0u, 0u, 0u, 0u); };
      if (round > 0 && !__all_sync(0xffffffffu, mbar_wait_role(sm.qfree(), (round - 1) & 1, fail))) return false;
      float top = 0.f;
#pragma unroll 1
      for (int i = 0; i < 16; i += 4) {
        uint4 raw[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) raw[k] = chunk(i + k);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t v[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
          if (PAIR || stream == 0) sts128(chunk_at(sm.q(PAIR ? stream : 0, false), r, i + k), v[0], v[1], v[2], v[3]);
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(low(v[e])), fabsf(high(v[e]))));
        }
      }
      // 2^e with the largest element in [2^14, 2^15) 2^e
      const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 120) - 14;
      const float down = __uint_as_float((uint32_t)(127 - e) << 23);
      scale16 = scale * __uint_as_float((uint32_t)(127 + e) << 23);
      if (PAIR || stream == 1) {
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
          const uint4 raw = chunk(i);
          auto h = [&](uint32_t v) { return pack_f16(low(v) * down, high(v) * down); };
          sts128(chunk_at(sm.q(PAIR ? stream : 0, true), r, i), h(raw.x), h(raw.y), h(raw.z), h(raw.w));
        }
      }
      fence_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(sm.qfull());
      return true;
    };
    bool ok = true;
    // Round -1 only stages the first item's queries.
#pragma unroll 1
    for (int round = -1; ok; ++round) {
      if (round >= 0 && !x.valid) break;
      const int n = round >= 0 ? x.n() : 0;
      float ref = real ? -INFINITY : 0.f, sum = 0.f;
      bool careful = true;  // some row of the warp has no reference yet
      int it = 0;           // tiles of this item done by this stream
      const bool idle = !__any_sync(0xffffffffu, real);  // no row of the warp needs weights
#pragma unroll 1
      for (int u = PAIR ? 0 : stream; u < n; u += PAIR ? 1 : 2) {
        const int t = x.t0 + u;
        const bool codes = x.codes(t);
        ok = __all_sync(0xffffffffu, mbar_wait_role(sm.sfull(stream), tiles & 1, fail));
        if (!ok) break;
        tcgen05_after_sync();
        if (idle) {
          tcgen05_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(sm.pready(stream, 0)), mbar_arrive(sm.pready(stream, 1));
          ++it;
          ++tiles;
          continue;
        }
        const float sc = codes ? scale16 : scale;
        // keys of the tile that the row sees: all of them, or by the bits of `see`
        const int first = codes ? (t - 1 - x.hi_tiles) * kTile : (t - 1) * kTile;
        const int there = t == 0 ? 0 : (codes ? x.n_lo : x.n_hi) - first;  // keys of the tile
        const bool masked = t == 0 || there < kTile || (!codes && x.free_slot >= first && x.free_slot < first + kTile);
        auto see = [&](int word) {  // 32 keys
          if (t == 0) return word == 0 ? mask[0] : word == 1 ? mask[1] : word == 2 ? mask[2] : mask[3];
          const int left = there - 32 * word;
          uint32_t bits = left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
          if (!codes && ((x.free_slot - first) >> 5) == word) bits &= ~(1u << ((x.free_slot - first) & 31));
          return bits;
        };
        // Both halves of the keys or, where the rows stand twice, the copy's: its other weights are 0.
#pragma unroll 1
        for (int half = upper ? 1 : 0; half < (twin && !upper ? 1 : 2); ++half) {
          float v[64];
          uint32_t w[32];
          auto load = [&]() {
            tmem_ld32(ts + 64 * half, v);
            tmem_ld32(ts + 64 * half + 32, v + 32);
            tmem_wait_ld(v);
            reg_fence(v + 32);
          };
          // weights of the scores in v, packed, and their sum
          auto weigh_as = [&](float less, auto f16) {
            const uint64_t s2 = f32x2(sc, sc), r2 = f32x2(-less, -less);
            uint64_t acc[2] = {0ull, 0ull};
#pragma unroll
            for (int i = 0; i < 64; i += 2) {
              float y0, y1;
              f32x2_split(fma_f32x2(f32x2(v[i], v[i + 1]), s2, r2), y0, y1);
              y0 = fast_exp2(y0), y1 = fast_exp2(y1);
              acc[(i >> 1) & 1] = add_f32x2(acc[(i >> 1) & 1], f32x2(y0, y1));
              w[i >> 1] = flash::pack16<decltype(f16)::value>(y0, y1);
            }
            float s0, s1;
            f32x2_split(add_f32x2(acc[0], acc[1]), s0, s1);
            return s0 + s1;
          };
          auto weigh = [&](float less) {
            return codes ? weigh_as(less, std::true_type{}) : weigh_as(less, std::false_type{});
          };
          // Without masks and with a reference in every row the weights come first and their sum tells whether a reference
          // was too low (or a score NaN); then, or else at once: masks, the largest score, a moved reference with O rescaled.
          bool slow = masked || careful;
#pragma unroll 1
          while (true) {
            load();
            if (slow) {
              if (masked) {
                const uint32_t s0 = see(2 * half), s1 = see(2 * half + 1);
                flash::mask_scores(v, s0, -INFINITY);
                flash::mask_scores(v + 32, s1, -INFINITY);
              }
              float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
              for (int i = 0; i < 64; i += 4) {
                mx[0] = flash::max3(mx[0], v[i], v[i + 1]);
                mx[1] = flash::max3(mx[1], v[i + 2], v[i + 3]);
              }
              const float largest = fmaxf(mx[0], mx[1]) * sc;
              const float next = largest > ref + kSlack ? largest - kDrop : ref;
              const bool moves = next != ref && ref != -INFINITY;
              if (__any_sync(0xffffffffu, moves)) {
                const float f = moves ? fast_exp2(ref - next) : 1.f;
                const bool same = half && !twin;  // the last product in O: the first half of this tile, or the tile before
                if (same || it > 0) {
                  ok = __all_sync(0xffffffffu, mbar_wait_role(sm.odone(stream, same ? 0 : 1), (same ? tiles : tiles - 1) & 1, fail));
                  if (!ok) break;
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
              careful = __any_sync(0xffffffffu, ref == -INFINITY);
            }
            const float got = weigh(ref == -INFINITY ? 0.f : ref);
            if (slow || __all_sync(0xffffffffu, got <= kSumMax)) {
              sum += got;
              break;
            }
            slow = true;
          }
          if (!ok) break;
          tmem_st32(ts + 32 * half, w);  // (over columns of S that both halves have left)
          if (twin) {
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = 0u;
            tmem_st32(ts + 32 * (half ^ 1), w);
          }
          tmem_wait_st();
          tcgen05_before_sync();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(sm.pready(stream, half));
            if (twin) mbar_arrive(sm.pready(stream, half ^ 1));
          }
        }
        if (!ok) break;
        ++it;
        ++tiles;
      }
      // where the row goes; the next item's queries are staged before this one is written
      const bool live = real, whole = x.slot < 0;
      const bool there = !upper && (PAIR ? 2 * x.m_block + stream : x.m_block) * kTile + row < p.rows;
      const size_t part_at = (size_t)max(x.slot, 0) * L::kItemRows + (PAIR ? stream * kTile : 0) + row;
      const long long out_at = x.b * a.out.b + head * a.out.h + node * a.out.t;
      const size_t lse_at = ((size_t)x.b * a.heads_q + head) * a.nodes + node;
      bool poisoned = false;
      const bool nodes_here = x.t0 == 0;
      uint32_t old_mask[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) old_mask[i] = mask[i];
      if (ok) ok = next_item(round + 1, x);
      if (ok && x.valid) ok = stage_rows(round + 1);
      if (round < 0) {
        if (!PAIR) ok = !group_sync<1, kSoftThreads>(!ok);  // (all of them go on, or none)
        continue;
      }
      if (ok && it > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait_role(sm.odone(stream, 1), (tiles - 1) & 1, fail));
        tcgen05_after_sync();
      }
      if constexpr (!PAIR) {
        s_part[(2 * stream) * kTile + r] = it > 0 ? ref : -INFINITY;
        s_part[(2 * stream + 1) * kTile + r] = it > 0 ? sum : 0.f;
        tcgen05_before_sync();
        if (group_sync<1, kSoftThreads>(!ok || *fail)) break;  // (both streams' products are done)
        tcgen05_after_sync();
      } else if (!ok) {
        break;
      }
      if (nodes_here) {
#pragma unroll
        for (int i = 0; i < 4; ++i) poisoned |= (old_mask[i] & s_bad[round % kBadRing][i]) != 0u;
      }
      float top = ref, total = sum, g0 = 1.f, g1 = 0.f;
      if constexpr (!PAIR) {
        const int other = twin ? r ^ (kTile / 2) : r;  // the row's other copy
        const float m0 = s_part[r], m1 = s_part[2 * kTile + r];
        top = fmaxf(m0, m1);
        if (twin) top = fmaxf(top, fmaxf(s_part[other], s_part[2 * kTile + other]));
        auto factor = [&](float m) { return m == -INFINITY ? 0.f : fast_exp2(m - top); };
        g0 = factor(m0);
        g1 = factor(m1);
        total = s_part[kTile + r] * g0 + s_part[3 * kTile + r] * g1;
        // (added in the same order by both copies)
        const float rest = s_part[kTile + other] * factor(s_part[other]) + s_part[3 * kTile + other] * factor(s_part[2 * kTile + other]);
        if (twin) total = upper ? rest + total : total + rest;
      }
      const bool blank = !live || total == 0.f;
      const float lse2 = blank ? -INFINITY : top + log2f(total);
      const float inv = poisoned ? __int_as_float(0x7fffffff) : 1.f / total;
      g0 *= inv;
      g1 *= inv;
      char* dst = whole ? static_cast<char*>(a.out.p) + out_at * (a.out_f32 ? 4 : 2)
                        : reinterpret_cast<char*>(p.part_o + part_at * kHeadDim);
      const uint32_t o0 = PAIR ? to : tmem + 256 + lanes;
#pragma unroll 1
      for (int q = 0; q < (PAIR ? 4 : 2); ++q) {
        const int ch = 32 * (PAIR ? q : 2 * stream + q);
        float v[32];
        tmem_ld32(o0 + ch, v);
        tmem_wait_ld(v);
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = blank ? 0.f : v[e] * g0;
        if (!PAIR && n > 1) {
          float v1[32];
          tmem_ld32(o0 + 128 + ch, v1);
          tmem_wait_ld(v1);
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = blank ? 0.f : fmaf(v1[e], g1, v[e]);
        }
        if constexpr (!PAIR) {
          if (twin) {  // the upper copy's part goes to the lower one's thread
            float* ex = reinterpret_cast<float*>(smem_raw + (sm.exchange(stream) - smem_u32(smem_raw))) + row * kExPitch;
            if (upper) {
#pragma unroll
              for (int e = 0; e < 32; ++e) ex[e] = v[e];
            }
            group_sync<1, kSoftThreads>(false);
            if (!upper) {
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] += ex[e];
            }
            group_sync<1, kSoftThreads>(false);
          }
        }
        if (there) flash::store_out32<false>(dst, !whole || a.out_f32, ch, v);
      }
      if (there && (PAIR || stream == 0)) {  // (upper copies are not there)
        if (!whole)
          p.part_lse[part_at] = lse2;
        else if (a.lse)
          a.lse[lse_at] = lse2 * kLn2;
      }
      if constexpr (!PAIR) {  // both warpgroups have read both O before the next item's products overwrite them
        tcgen05_before_sync();
        if (group_sync<1, kSoftThreads>(*fail)) break;
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

template <int BITS, bool PAIR>
cudaError_t launch_variant(const TreeKernelArgs& p, int grid, cudaStream_t st) {
  static std::atomic<uint64_t> configured;  // one bit per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev > 63 || !(configured.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(tree_kernel<BITS, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<PAIR>::kSmem);
    if (e != cudaSuccess) return e;
    configured.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch_chained(tree_kernel<BITS, PAIR>, dim3(grid), dim3(kThreads), Layout<PAIR>::kSmem, st, p);
}

}  // namespace tree
}  // namespace mikv
