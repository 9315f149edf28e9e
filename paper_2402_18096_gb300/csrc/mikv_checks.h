// mikv_checks.h — argument checks that the entry points of the C ABI share (host only): cache shapes and arrays, strided
// views, alignments.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "mikv_device.cuh"
#include "mikv_internal.h"

namespace mikv {

inline mikv_status cuda_status(cudaError_t e) { return e == cudaSuccess ? MIKV_OK : MIKV_ERR_CUDA; }

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline bool positive(float x) { return x > 0.f && x <= 3.402823466e38f; }

inline bool shape_ok(const mikv_shape* s) {
  return s && s->batch > 0 && s->heads_q > 0 && s->heads_kv > 0 && s->heads_q % s->heads_kv == 0 &&
         s->head_dim > 0 && s->bits >= 0 && (s->bits == 0 || s->group > 0) && s->hi_cap >= 0 &&
         s->hi_stride >= s->hi_cap &&
         s->hi_stride % 16 == 0 && s->lo_cap >= 0 && s->lo_cap % 16 == 0;
}

inline mikv_status shape_supported(const mikv_shape* s) {
  if (!shape_ok(s)) return MIKV_ERR_ARG;
  const int G = s->heads_q / s->heads_kv;
  if (s->head_dim != kHeadDimH) return MIKV_ERR_UNSUPPORTED;
  if (s->bits != 0) {  // bits == 0: eviction, no retained set (its group is ignored)
    if (s->bits < 2 || s->bits > 4) return MIKV_ERR_UNSUPPORTED;
    if (s->group != 32 && s->group != 64 && s->group != 128) return MIKV_ERR_UNSUPPORTED;
  }
  if (G != 1 && G != 2 && G != 4 && G != 8) return MIKV_ERR_UNSUPPORTED;
  const int hb = s->hi_bits;
  if (hb != 0 && hb != 16 && hb != 8 && hb != 4 && hb != 2) return MIKV_ERR_UNSUPPORTED;
  if (hb != 0 && hb != 16 && s->hi_group != kHiGroup) return MIKV_ERR_UNSUPPORTED;
  if (s->k_channel_group != 0) {  // per-channel retained keys (App. C)
    if (s->k_channel_group != kKchGroup || (hb != 0 && hb != 16) || s->bits == 0) return MIKV_ERR_UNSUPPORTED;
    if (s->hi_stride < s->hi_cap + kKchGroup || s->lo_cap % kKchGroup) return MIKV_ERR_ARG;
  }
  return MIKV_OK;
}

// The cache's arrays exist (and, for a coded important set, so do its parameter arrays, 16-byte aligned).
inline bool cache_ok(const mikv_cache* c, const mikv_shape* s) {
  if (!(c && c->k_hi && c->v_hi && c->hi_tok && c->acc)) return false;
  if (!evicting(*s) && !(c->k_codes && c->v_codes && c->k_params && c->v_params && c->lo_tok)) return false;
  if (hi_bits_of(*s) != 16)
    return c->k_hi_params && c->v_hi_params && aligned(c->k_hi_params, 16) && aligned(c->v_hi_params, 16);
  return true;
}

inline int elem_bytes(int dtype) { return dtype == MIKV_F32 ? 4 : 2; }

constexpr int64_t kStrideMax = (int64_t)1 << 38;  // elements: a byte stride then fits a tensor map's 40 bits

// Strides of the dimensions that are there lie in [least, kStrideMax); unused ones become 0.
inline bool strides_of(const mikv_view* x, int64_t batch, int64_t heads, int64_t tokens, int64_t least, long long (&s)[3]) {
  const int64_t n[3] = {batch, heads, tokens}, st[3] = {x->stride_batch, x->stride_head, x->stride_token};
  for (int i = 0; i < 3; ++i) {
    s[i] = n[i] == 1 ? 0 : st[i];
    if (n[i] != 1 && (st[i] < least || st[i] >= kStrideMax)) return false;
  }
  return true;
}

// Attention operands: 16-byte aligned data and strides; a zero batch or head stride only where `shared` allows it.
inline mikv_status attn_view(const mikv_view* x, int64_t batch, int64_t heads, int64_t tokens, int bytes, bool shared,
                      long long (&s)[3]) {
  if (!x || !x->data || !aligned(x->data, 16)) return MIKV_ERR_ARG;
  if (!strides_of(x, batch, heads, tokens, 0, s)) return MIKV_ERR_ARG;
  const int64_t n[3] = {batch, heads, tokens};
  for (int i = 0; i < 3; ++i) {
    if (s[i] * bytes % 16) return MIKV_ERR_ARG;
    if (n[i] != 1 && s[i] == 0 && !(shared && i < 2)) return MIKV_ERR_ARG;
  }
  return MIKV_OK;
}

}  // namespace mikv
