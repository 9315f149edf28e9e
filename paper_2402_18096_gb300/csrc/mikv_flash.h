// mikv_flash.h — arguments of the attention kernels over bf16 / fp16 keys (mikv_flash.cu): prompts and shared
// prefixes.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mikv_device.cuh"

namespace mikv {

// Both entry points are one problem to the kernels: `batch` sets of keys, each attended by tq "tokens" of G query
// heads per KV head. For a prompt a token is a query position; for a shared prefix it is one of its requests.
struct FlashArgs {
  const void *q, *k, *v;
  long long q_b, q_h, q_t, k_b, k_h, k_t, v_b, v_h, v_t;  // element strides
  void* out;
  long long o_b, o_h, o_t;
  float* stat;                 // log-sum-exp (stat_pair 0), or (log-sum-exp, 1) pairs (stat_pair 1), or nullptr
  long long s_b, s_h, s_t;     // strides of stat in entries
  int stat_pair;
  const float* own_out;        // join: [batch * tq][heads_q][128] with its (max, sum), or nullptr
  const float* own_ml;
  const int2* spans;           // [batch][tq], or nullptr
  const int32_t* lens;         // [batch] visible keys, or nullptr
  const int32_t* pos;          // [batch][tq] query positions, or nullptr
  const float* slopes;         // [heads_q] or nullptr
  int batch, tq, tk, heads_q, heads_kv, G;
  int causal, q_start;
  int pos_at_len;              // without `pos`: 1 = a query stands at its set's length, 0 = at q_start + token
  float sm_scale, softcap;
  int* status;
};

// Division of 0 <= n < 2^31 by d > 0 through a multiplication: with s = ceil(log2 d) and mul = ceil(2^(31 + s) / d),
// mul exceeds 2^(31 + s) / d by less than 1, so n mul / 2^(31 + s) exceeds n / d by less than 2^-s <= 1 / d.
struct FastDiv {
  int d;
  unsigned mul, shift;
  void set(int by) {
    d = by;
    shift = 0;
    while ((1ll << shift) < by) ++shift;
    mul = (unsigned)(((1ull << (31 + shift)) + by - 1) / by);
  }
#ifdef __CUDACC__
  __device__ __forceinline__ int div(int n) const {
    return (int)(((unsigned long long)(unsigned)n * mul) >> (31 + shift));
  }
#endif
};

// What the tensor-core kernel takes: the problem, its tensor maps, and its share of the work plan.
struct FlashKernelArgs {
  CUtensorMap map_q;    // [batch][tokens][heads][128], box 64 channels x G heads x 128 / G tokens, 128B swizzle
  CUtensorMap map_k, map_v;  // [batch][heads][keys][128], box 64 channels x 128 keys
  FlashArgs a;
  int k_batch, k_head, v_batch, v_head;  // 1, or 0 where the dimension is shared (zero stride)
  int m_blocks;         // row tiles (pairs) of one KV head
  int n_items;          // batch * heads_kv * m_blocks
  int group_heads;      // (set, KV head) combinations whose items are worked on together
  int log2_G;
  // an item's number taken apart: by group, by rank within a full or the last group, and a head into its set
  FastDiv by_group, by_rank, by_last, by_head;
  int out_f32;          // the output is fp32; else of the keys' type
  // Shares: the key tiles of all row tiles, end to end, in equal runs for the CTAs.
  int shares;           // 0: whole row tiles
  int by_length;        // units of a row tile: the tiles of its set's length (lens), else `units`
  int units;
  int share_each, share_extra;         // (not by_length) units of a CTA, and how many CTAs have one more
  float inv_units;                     // 1 / units
  FastDiv by_units, by_set, by_block;  // a unit into its row tile, a row tile into its set, and into its head
  int2* part_table;     // [batch * heads_kv * m_blocks]: first CTA of a row tile, and the number of its parts
  float* part_o;        // [slots][rows of an item][128] normalised outputs, slot = CTA + row tile
  float* part_lse;      // [slots][rows of an item] log2 of the sum of 2^x (-inf: nothing seen)
};

size_t flash_workspace_bytes(int batch, int heads_kv, int G, int tq, int tk, int num_sms);
bool flash_fits(int batch, int heads_kv, int G, int tq);  // the number of items stays in range
cudaError_t launch_flash(const FlashArgs& a, bool f16, bool out_f32, void* ws, int num_sms, cudaStream_t st);

}  // namespace mikv
