// mikv_abi_tree.cu — host side of the entry points for drafted tokens (include/mikv.h): argument validation and
// dispatch. Nothing here allocates device memory or synchronises.
#include <cuda_runtime.h>
#include <string.h>

#include <atomic>
#include <new>
#include <vector>

#include "../../include/mikv.h"
#include "mikv_checks.h"
#include "mikv_nvtx.h"
#include "mikv_tree.h"

using namespace mikv;

namespace {

// SMs of the current device (asked once per device).
int num_sms() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 148;
  if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 148;
  if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

// Shapes these kernels take: a bf16 important set, per-token retained keys.
mikv_status drafts_supported(const mikv_shape* s) {
  const mikv_status st = shape_supported(s);
  if (st != MIKV_OK) return st;
  if (hi_bits_of(*s) != 16 || kch_of(*s)) return MIKV_ERR_UNSUPPORTED;
  return (int64_t)s->batch * s->heads_kv > 65535 ? MIKV_ERR_UNSUPPORTED : MIKV_OK;
}

// The arrays that these kernels read in 16-byte pieces.
bool cache_aligned(const mikv_cache* c, const mikv_shape* s) {
  if (!aligned(c->k_hi, 16) || !aligned(c->v_hi, 16) || !aligned(c->hi_tok, 4) || !aligned(c->acc, 4) ||
      !aligned(c->balancer, 16))
    return false;
  return evicting(*s) || (aligned(c->k_codes, 16) && aligned(c->v_codes, 16) && aligned(c->k_params, 16) &&
                          aligned(c->v_params, 16) && aligned(c->lo_tok, 4));
}

mikv_status held_of(const mikv_lengths* lens, const mikv_shape* s, HeldArgs& held) {
  held = HeldArgs{};
  held.hi_cap = s->hi_cap;
  if (!lens) return MIKV_OK;
  if (!aligned(lens->n_hi, 4) || !aligned(lens->n_lo, 4) || !aligned(lens->slots, 4) || lens->n_lo_max < 0)
    return MIKV_ERR_ARG;
  if (evicting(*s) ? lens->n_lo_max > 0 : lens->n_lo_max > s->lo_cap) return MIKV_ERR_ARG;
  held.n_hi = lens->n_hi, held.n_lo = lens->n_lo, held.slots = lens->slots;
  held.n_lo_max = lens->n_lo_max;
  return MIKV_OK;
}

mikv_status view_of(const mikv_view* x, int64_t batch, int64_t heads, int64_t nodes, int bytes, TreeView& v) {
  long long s[3];
  const mikv_status st = attn_view(x, batch, heads, nodes, bytes, false, s);
  if (st == MIKV_OK) v = {x->data, s[0], s[1], s[2]};
  return st;
}

bool nodes_ok(int32_t n) { return n >= 1 && n <= kTreeNodes; }

// The row `to` of every pair once, and none of `from` among them where `same`; where the lengths alone are `joint`, none but a
// row that stays itself.
mikv_status pairs_ok(const int32_t* pairs, int32_t n, int32_t batch, int32_t to_batch, bool same, bool joint) {
  std::vector<uint8_t> role;
  try {
    role.assign((size_t)(to_batch > batch ? to_batch : batch), 0);
  } catch (const std::bad_alloc&) {
    return MIKV_ERR_ARG;
  }
  for (int32_t i = 0; i < n; ++i) {
    const int32_t from = pairs[2 * i], to = pairs[2 * i + 1];
    if (from < 0 || from >= batch || to < 0 || to >= to_batch || (role[to] & 1)) return MIKV_ERR_ARG;
    role[to] |= from == to ? 3 : 1;
  }
  for (int32_t i = 0; (same || joint) && i < n; ++i) {
    const uint8_t r = role[pairs[2 * i]];
    if (same ? (r & 1) != 0 : r == 1) return MIKV_ERR_ARG;
  }
  return MIKV_OK;
}

bool copy_aligned(const mikv_cache* c, const mikv_shape* s) {
  const void* all[] = {c->k_hi,    c->v_hi,     c->hi_tok,   c->acc,    c->k_codes, c->v_codes,
                       c->k_params, c->v_params, c->lo_tok};
  for (const void* p : all)
    if (!aligned(p, 16)) return false;
  return hi_bits_of(*s) == 16 || (aligned(c->k_hi_params, 16) && aligned(c->v_hi_params, 16));
}

}  // namespace

extern "C" {

mikv_status mikv_tree_masks(uint32_t* masks, int32_t* positions, const int32_t* parents, int32_t batch, int32_t nodes,
                            const int32_t* first, int32_t start, void* stream) {
  MIKV_CALL_RANGE();
  if (!masks || !parents || batch <= 0 || nodes <= 0 || !aligned(masks, 16) || !aligned(positions, 4) ||
      !aligned(parents, 4) || !aligned(first, 4))
    return MIKV_ERR_ARG;
  if (!nodes_ok(nodes)) return MIKV_ERR_UNSUPPORTED;
  return cuda_status(launch_tree_masks(reinterpret_cast<uint4*>(masks), positions, parents, batch, nodes, first, start,
                                       static_cast<cudaStream_t>(stream)));
}

size_t mikv_tree_workspace_bytes(const mikv_shape* shape, int32_t nodes) {
  if (drafts_supported(shape) != MIKV_OK || !nodes_ok(nodes) || !tree_sizes_ok(*shape, nodes)) return 0;
  return tree_workspace_bytes(*shape, nodes, num_sms());
}

mikv_status mikv_tree_attention(const mikv_shape* shape, const mikv_cache* cache, const mikv_tree_desc* d,
                                const uint32_t* masks, const mikv_view* q, const mikv_view* k, const mikv_view* v,
                                const mikv_view* out, const mikv_lengths* lens, float* lse, void* workspace,
                                size_t ws_bytes, void* stream) {
  MIKV_CALL_RANGE();
  mikv_status st = drafts_supported(shape);
  if (st != MIKV_OK) return st;
  if (!d || !cache_ok(cache, shape) || !cache_aligned(cache, shape) || !masks || !aligned(masks, 16) || !aligned(lse, 4))
    return MIKV_ERR_ARG;
  if (d->nodes <= 0 || !positive(d->sm_scale) || (d->out_dtype != MIKV_BF16 && d->out_dtype != MIKV_F32))
    return MIKV_ERR_ARG;
  if (!nodes_ok(d->nodes) || !tree_sizes_ok(*shape, d->nodes)) return MIKV_ERR_UNSUPPORTED;
  TreeArgs a;
  memset(&a, 0, sizeof a);
  if ((st = view_of(q, shape->batch, shape->heads_q, d->nodes, 2, a.q)) != MIKV_OK) return st;
  if ((st = view_of(k, shape->batch, shape->heads_kv, d->nodes, 2, a.k)) != MIKV_OK) return st;
  if ((st = view_of(v, shape->batch, shape->heads_kv, d->nodes, 2, a.v)) != MIKV_OK) return st;
  if ((st = view_of(out, shape->batch, shape->heads_q, d->nodes, elem_bytes(d->out_dtype), a.out)) != MIKV_OK) return st;
  if ((st = held_of(lens, shape, a.held)) != MIKV_OK) return st;
  if (!workspace || !aligned(workspace, 256) || ws_bytes < mikv_tree_workspace_bytes(shape, d->nodes))
    return MIKV_ERR_WORKSPACE;
  a.k_hi = static_cast<const __nv_bfloat16*>(cache->k_hi);
  a.v_hi = static_cast<const __nv_bfloat16*>(cache->v_hi);
  a.k_codes = static_cast<const uint8_t*>(cache->k_codes);
  a.v_codes = static_cast<const uint8_t*>(cache->v_codes);
  a.k_params = static_cast<const __half2*>(cache->k_params);
  a.v_params = static_cast<const __half2*>(cache->v_params);
  a.balancer = cache->balancer;
  a.masks = reinterpret_cast<const uint4*>(masks);
  a.lse = lse;
  a.status = static_cast<int*>(workspace);
  a.batch = shape->batch, a.heads_q = shape->heads_q, a.heads_kv = shape->heads_kv;
  a.G = shape->heads_q / shape->heads_kv;
  a.nodes = d->nodes;
  a.hi_stride = shape->hi_stride, a.lo_cap = shape->lo_cap;
  a.bits = lo_bits_of(*shape), a.group = lo_group_of(*shape);
  a.sm_scale = d->sm_scale;
  a.out_f32 = d->out_dtype == MIKV_F32;
  return cuda_status(launch_tree(a, workspace, num_sms(), static_cast<cudaStream_t>(stream)));
}

mikv_status mikv_path_importance(const mikv_shape* shape, const mikv_cache* cache, int32_t nodes, float sm_scale,
                                 const int32_t* path, int32_t steps, const mikv_view* q, const mikv_view* k,
                                 const float* lse, const mikv_lengths* lens, float* gained, void* stream) {
  MIKV_CALL_RANGE();
  mikv_status st = drafts_supported(shape);
  if (st != MIKV_OK) return st;
  if (!cache_ok(cache, shape) || !cache_aligned(cache, shape) || !path || !lse || !gained || nodes <= 0 || steps <= 0 ||
      !positive(sm_scale) || !aligned(path, 4) || !aligned(lse, 4) || !aligned(gained, 4))
    return MIKV_ERR_ARG;
  if (!nodes_ok(nodes) || !nodes_ok(steps)) return MIKV_ERR_UNSUPPORTED;
  PathArgs a;
  memset(&a, 0, sizeof a);
  if ((st = view_of(q, shape->batch, shape->heads_q, nodes, 2, a.q)) != MIKV_OK) return st;
  if ((st = view_of(k, shape->batch, shape->heads_kv, nodes, 2, a.k)) != MIKV_OK) return st;
  if ((st = held_of(lens, shape, a.held)) != MIKV_OK) return st;
  a.cache = cache;
  a.path = path, a.lse = lse, a.gained = gained;
  a.steps = steps, a.nodes = nodes;
  a.sm_scale = sm_scale;
  return cuda_status(launch_path_importance(*shape, a, static_cast<cudaStream_t>(stream)));
}

size_t mikv_commit_workspace_bytes(const mikv_shape* shape, int32_t steps) {
  return drafts_supported(shape) != MIKV_OK || !nodes_ok(steps) ? 0 : kWsHeader;
}

mikv_status mikv_commit_path(const mikv_shape* shape, const mikv_cache* cache, int32_t nodes, const int32_t* path,
                             int32_t steps, const mikv_view* k, const mikv_view* v, const float* gained,
                             const int32_t* first, const mikv_lengths* lens, const mikv_lengths* lens_out,
                             int32_t* next, void* workspace, size_t ws_bytes, void* stream) {
  MIKV_CALL_RANGE();
  mikv_status st = drafts_supported(shape);
  if (st != MIKV_OK) return st;
  if (!cache_ok(cache, shape) || !cache_aligned(cache, shape) || !path || !gained || !first || !lens || nodes <= 0 ||
      steps <= 0 || !aligned(path, 4) || !aligned(gained, 4) || !aligned(first, 4) || !aligned(next, 4))
    return MIKV_ERR_ARG;
  if (lens_out && (!aligned(lens_out->n_hi, 4) || !aligned(lens_out->n_lo, 4))) return MIKV_ERR_ARG;
  if (!nodes_ok(nodes) || !nodes_ok(steps)) return MIKV_ERR_UNSUPPORTED;
  PathArgs a;
  memset(&a, 0, sizeof a);
  if ((st = view_of(k, shape->batch, shape->heads_kv, nodes, 2, a.k)) != MIKV_OK) return st;
  if ((st = view_of(v, shape->batch, shape->heads_kv, nodes, 2, a.v)) != MIKV_OK) return st;
  if ((st = held_of(lens, shape, a.held)) != MIKV_OK) return st;
  if (!workspace || !aligned(workspace, 256) || ws_bytes < mikv_commit_workspace_bytes(shape, steps))
    return MIKV_ERR_WORKSPACE;
  a.cache = cache;
  a.path = path, a.gained = const_cast<float*>(gained), a.first = first;
  if (lens_out) a.n_hi_out = lens_out->n_hi, a.n_lo_out = lens_out->n_lo;
  a.next = next;
  a.status = static_cast<int*>(workspace);
  a.steps = steps, a.nodes = nodes;
  return cuda_status(launch_commit(*shape, a, static_cast<cudaStream_t>(stream)));
}

mikv_status mikv_copy_requests(const mikv_shape* shape, const mikv_cache* cache, const mikv_shape* to_shape,
                               const mikv_cache* to_cache, const int32_t* pairs, int32_t n, const mikv_lengths* lens,
                               const mikv_lengths* to_lens, void* stream) {
  MIKV_CALL_RANGE();
  mikv_status st = shape_supported(shape);
  if (st != MIKV_OK) return st;
  if ((st = shape_supported(to_shape)) != MIKV_OK) return st;
  if (!cache_ok(cache, shape) || !cache_ok(to_cache, to_shape) || !copy_aligned(cache, shape) ||
      !copy_aligned(to_cache, to_shape) || n < 0 || (n > 0 && !pairs))
    return MIKV_ERR_ARG;
  const mikv_shape &x = *shape, &y = *to_shape;
  if (x.heads_kv != y.heads_kv || x.bits != y.bits || (x.bits && x.group != y.group) || hi_bits_of(x) != hi_bits_of(y) ||
      x.k_channel_group != y.k_channel_group)
    return MIKV_ERR_ARG;
  if (x.heads_kv > 65535) return MIKV_ERR_UNSUPPORTED;
  HeldArgs held;
  if ((st = held_of(lens, shape, held)) != MIKV_OK) return st;
  if (to_lens && (!aligned(to_lens->n_hi, 4) || !aligned(to_lens->n_lo, 4) || !aligned(to_lens->slots, 4) ||
                  (to_lens->slots && !held.slots)))
    return MIKV_ERR_ARG;
  const bool counted_hi = held.n_hi || (to_lens && to_lens->n_hi);  // else every slot of the target counts as in use
  if (y.hi_cap < x.hi_cap || ((kch_of(x) || !counted_hi) && y.hi_cap != x.hi_cap) ||
      (!evicting(x) && y.lo_cap < held.n_lo_max))
    return MIKV_ERR_CAPACITY;
  // the caches are one or share nothing: of one, all arrays are the same
  const void* from_all[] = {cache->k_hi, cache->v_hi, cache->hi_tok, cache->acc, cache->k_codes, cache->v_codes,
                            cache->k_params, cache->v_params, cache->lo_tok, cache->k_hi_params, cache->v_hi_params};
  const void* to_all[] = {to_cache->k_hi, to_cache->v_hi, to_cache->hi_tok, to_cache->acc, to_cache->k_codes,
                          to_cache->v_codes, to_cache->k_params, to_cache->v_params, to_cache->lo_tok,
                          to_cache->k_hi_params, to_cache->v_hi_params};
  const int arrays = hi_bits_of(x) == 16 ? (evicting(x) ? 4 : 9) : 11;
  int shared = 0, counted = 0;
  for (int i = 0; i < arrays; ++i)
    if (!evicting(x) || i < 4 || i > 8) ++counted, shared += from_all[i] == to_all[i];
  if (shared != 0 && shared != counted) return MIKV_ERR_ARG;
  const bool same = shared != 0;
  if (same && (x.hi_stride != y.hi_stride || x.lo_cap != y.lo_cap)) return MIKV_ERR_ARG;
  const bool joint = lens && to_lens && ((lens->n_hi && lens->n_hi == to_lens->n_hi) || (lens->n_lo && lens->n_lo == to_lens->n_lo) ||
                                         (lens->slots && lens->slots == to_lens->slots));
  if ((st = pairs_ok(pairs, n, x.batch, y.batch, same, joint)) != MIKV_OK) return st;
  if (n == 0) return MIKV_OK;
  CopyLengths len = {held.n_hi, held.n_lo, held.slots, nullptr, nullptr, nullptr, held.n_lo_max};
  if (to_lens) len.to_n_hi = to_lens->n_hi, len.to_n_lo = to_lens->n_lo, len.to_slots = to_lens->slots;
  return cuda_status(launch_copy_requests(x, *cache, y, *to_cache, pairs, n, len, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
