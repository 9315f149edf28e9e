// mikv_abi_prompt.cu — host side of the prompt and shared-prefix entry points (include/mikv.h): argument
// validation and kernel dispatch. Nothing here allocates device memory or synchronises.
#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>
#include <string.h>

#include <atomic>

#include "../../include/mikv.h"
#include "mikv_flash.h"
#include "mikv_nvtx.h"
#include "mikv_rotary.h"

using namespace mikv;

namespace {

mikv_status cuda_status(cudaError_t e) { return e == cudaSuccess ? MIKV_OK : MIKV_ERR_CUDA; }

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

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int elem_bytes(int dtype) { return dtype == MIKV_F32 ? 4 : 2; }

constexpr int64_t kStrideMax = (int64_t)1 << 38;  // elements: a byte stride then fits a tensor map's 40 bits

// Strides of the dimensions that are there lie in [least, kStrideMax); unused ones become 0.
bool strides_of(const mikv_view* x, int64_t batch, int64_t heads, int64_t tokens, int64_t least, long long (&s)[3]) {
  const int64_t n[3] = {batch, heads, tokens}, st[3] = {x->stride_batch, x->stride_head, x->stride_token};
  for (int i = 0; i < 3; ++i) {
    s[i] = n[i] == 1 ? 0 : st[i];
    if (n[i] != 1 && (st[i] < least || st[i] >= kStrideMax)) return false;
  }
  return true;
}

// Attention operands: 16-byte aligned data and strides; a zero batch or head stride only where `shared` allows it.
mikv_status attn_view(const mikv_view* x, int64_t batch, int64_t heads, int64_t tokens, int bytes, bool shared,
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

bool positive(float x) { return x > 0.f && x <= 3.402823466e38f; }

mikv_status attn_common(int32_t dtype, int32_t out_dtype, int32_t batch, int32_t heads_q, int32_t heads_kv,
                        int32_t head_dim, int32_t tq, int32_t tk, float sm_scale, float softcap) {
  if (batch <= 0 || heads_q <= 0 || heads_kv <= 0 || heads_q % heads_kv || tq <= 0 || tk < 0) return MIKV_ERR_ARG;
  if (dtype != MIKV_BF16 && dtype != MIKV_F16) return MIKV_ERR_ARG;
  if (out_dtype != dtype && out_dtype != MIKV_F32) return MIKV_ERR_ARG;
  if (!positive(sm_scale) || !(softcap == 0.f || positive(softcap))) return MIKV_ERR_ARG;
  if (head_dim != kHeadDim) return MIKV_ERR_UNSUPPORTED;
  const int G = heads_q / heads_kv;
  if (G != 1 && G != 2 && G != 4 && G != 8) return MIKV_ERR_UNSUPPORTED;
  if (batch > 65535 || heads_q > 65535 || tk > INT_MAX - 512 || tq > INT_MAX / 8 - 512 ||
      !flash_fits(batch, heads_kv, G, tq))
    return MIKV_ERR_UNSUPPORTED;
  return MIKV_OK;
}

mikv_status prompt_ok(const mikv_prompt_desc* d) {
  if (!d) return MIKV_ERR_ARG;
  if (d->q_start > (1 << 30) || d->q_start < -(1 << 30)) return MIKV_ERR_UNSUPPORTED;  // (positions stay in 32 bits)
  return attn_common(d->dtype, d->out_dtype, d->batch, d->heads_q, d->heads_kv, d->head_dim, d->tq, d->tk, d->sm_scale,
                     d->softcap);
}

mikv_status prefix_ok(const mikv_prefix_desc* d) {
  if (!d || d->groups <= 0 || d->batch <= 0 || d->batch % d->groups) return MIKV_ERR_ARG;
  return attn_common(d->dtype, d->out_dtype, d->groups, d->heads_q, d->heads_kv, d->head_dim, d->batch / d->groups,
                     d->length, d->sm_scale, d->softcap);
}

}  // namespace

extern "C" {

mikv_status mikv_rotary_phases(const double* freq, int32_t n, uint64_t* phases) {
  if (!freq || !phases || n <= 0) return MIKV_ERR_ARG;
  for (int i = 0; i < n; ++i) {
    if (!(freq[i] >= 0.0 && freq[i] <= 1.7976931348623157e308)) return MIKV_ERR_ARG;
    const double turns = freq[i] / 6.283185307179586476925286766559;
    const double frac = turns - floor(turns);  // < 1, or 1 by rounding: a whole turn
    const double scaled = rint(ldexp(frac, 64));
    phases[i] = scaled >= 18446744073709551616.0 ? 0 : (uint64_t)scaled;
  }
  return MIKV_OK;
}

mikv_status mikv_rotary(const mikv_rotary_desc* d, const mikv_view* q_in, const mikv_view* q_out,
                        const mikv_view* k_in, const mikv_view* k_out, const uint64_t* phases,
                        const int32_t* positions, int32_t start, void* stream) {
  MIKV_CALL_RANGE();
  if (!d || !phases || !aligned(phases, 8) || !aligned(positions, 4)) return MIKV_ERR_ARG;
  if (d->dtype != MIKV_BF16 && d->dtype != MIKV_F16 && d->dtype != MIKV_F32) return MIKV_ERR_ARG;
  if (d->batch <= 0 || d->tokens < 0 || d->heads_q <= 0 || d->heads_k < 0) return MIKV_ERR_ARG;
  if (d->layout != MIKV_ROTARY_HALF && d->layout != MIKV_ROTARY_INTERLEAVED) return MIKV_ERR_ARG;
  if (d->rot < 2 || d->rot % 2 || d->rot > d->head_dim || !(fabsf(d->amplitude) <= 3.402823466e38f)) return MIKV_ERR_ARG;
  if (d->head_dim != kHeadDim || d->batch > 65535 || (int64_t)d->heads_q + d->heads_k > 65535) return MIKV_ERR_UNSUPPORTED;
  if (d->tokens == 0) return MIKV_OK;  // (an empty tensor may have no address)
  RotaryArgs a;
  memset(&a, 0, sizeof a);
  const int bytes = elem_bytes(d->dtype), n = 16 / bytes;
  bool vec = (d->layout == MIKV_ROTARY_HALF ? d->rot / 2 : d->rot) % n == 0 && (d->head_dim - d->rot) % n == 0;
  const mikv_view* in[2] = {q_in, k_in};
  const mikv_view* out[2] = {q_out, k_out};
  const int heads[2] = {d->heads_q, d->heads_k};
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0) continue;
    RotaryTensor& x = a.x[i];
    long long s[3], o[3];
    if (!in[i] || !out[i] || !in[i]->data || !out[i]->data || !aligned(in[i]->data, bytes) ||
        !aligned(out[i]->data, bytes))
      return MIKV_ERR_ARG;
    if (!strides_of(in[i], d->batch, heads[i], d->tokens, 0, s)) return MIKV_ERR_ARG;
    if (!strides_of(out[i], d->batch, heads[i], d->tokens, 1, o)) return MIKV_ERR_ARG;
    x = {in[i]->data, out[i]->data, s[0], s[1], s[2], o[0], o[1], o[2], heads[i]};
    vec = vec && aligned(x.in, 16) && aligned(x.out, 16);
    for (int j = 0; j < 3; ++j) vec = vec && s[j] % n == 0 && o[j] % n == 0;
  }
  a.phases = reinterpret_cast<const unsigned long long*>(phases);
  a.positions = positions;
  a.start = start;
  a.batch = d->batch;
  a.tokens = d->tokens;
  a.rot = d->rot;
  a.inverse = d->inverse != 0;
  a.amplitude = d->amplitude;
  return cuda_status(launch_rotary(a, d->dtype, d->layout, vec, static_cast<cudaStream_t>(stream)));
}

mikv_status mikv_mask_spans(int32_t* spans, int32_t batch, int32_t tq, int32_t tk, int32_t q_start, int32_t causal,
                            const int32_t* docs, int32_t n_docs, const int32_t* prefix, const int32_t* key_len,
                            void* stream) {
  MIKV_CALL_RANGE();
  if (!aligned(spans, 8) || batch <= 0 || tq < 0 || tk < 0 || (docs && n_docs <= 0)) return MIKV_ERR_ARG;
  if (!aligned(docs, 4) || !aligned(prefix, 4) || !aligned(key_len, 4)) return MIKV_ERR_ARG;
  if (batch > 65535 || n_docs == INT_MAX) return MIKV_ERR_UNSUPPORTED;
  if (tq == 0) return MIKV_OK;  // (an empty tensor may have no address)
  if (!spans) return MIKV_ERR_ARG;
  const SpanArgs a = {reinterpret_cast<int2*>(spans), docs, prefix, key_len, batch, tq, tk, q_start, causal, n_docs};
  return cuda_status(launch_mask_spans(a, static_cast<cudaStream_t>(stream)));
}

size_t mikv_prompt_workspace_bytes(const mikv_prompt_desc* d) {
  if (prompt_ok(d) != MIKV_OK) return 0;
  return flash_workspace_bytes(d->batch, d->heads_kv, d->heads_q / d->heads_kv, d->tq, d->tk, num_sms());
}

mikv_status mikv_prompt_attention(const mikv_prompt_desc* d, const mikv_view* q, const mikv_view* k,
                                  const mikv_view* v, const mikv_view* out, const int32_t* spans,
                                  const float* slopes, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  MIKV_CALL_RANGE();
  mikv_status st = prompt_ok(d);
  if (st != MIKV_OK) return st;
  if (!aligned(spans, 8) || !aligned(slopes, 4) || !aligned(lse, 4)) return MIKV_ERR_ARG;
  FlashArgs a;
  memset(&a, 0, sizeof a);
  long long s[3];
  if ((st = attn_view(q, d->batch, d->heads_q, d->tq, 2, false, s)) != MIKV_OK) return st;
  a.q = q->data, a.q_b = s[0], a.q_h = s[1], a.q_t = s[2];
  if ((st = attn_view(out, d->batch, d->heads_q, d->tq, elem_bytes(d->out_dtype), false, s)) != MIKV_OK) return st;
  a.out = out->data, a.o_b = s[0], a.o_h = s[1], a.o_t = s[2];
  if (d->tk > 0) {
    if ((st = attn_view(k, d->batch, d->heads_kv, d->tk, 2, true, s)) != MIKV_OK) return st;
    a.k = k->data, a.k_b = s[0], a.k_h = s[1], a.k_t = s[2];
    if ((st = attn_view(v, d->batch, d->heads_kv, d->tk, 2, true, s)) != MIKV_OK) return st;
    a.v = v->data, a.v_b = s[0], a.v_h = s[1], a.v_t = s[2];
  }
  if (!workspace || !aligned(workspace, 256) || ws_bytes < mikv_prompt_workspace_bytes(d)) return MIKV_ERR_WORKSPACE;
  a.stat = lse;
  a.s_b = (long long)d->heads_q * d->tq, a.s_h = d->tq, a.s_t = 1;
  a.spans = reinterpret_cast<const int2*>(spans);
  a.slopes = slopes;
  a.batch = d->batch, a.tq = d->tq, a.tk = d->tk;
  a.heads_q = d->heads_q, a.heads_kv = d->heads_kv, a.G = d->heads_q / d->heads_kv;
  a.causal = d->causal != 0;
  a.q_start = d->q_start;
  a.sm_scale = d->sm_scale, a.softcap = d->softcap;
  a.status = static_cast<int*>(workspace);
  return cuda_status(launch_flash(a, d->dtype == MIKV_F16, d->out_dtype == MIKV_F32, workspace, num_sms(),
                                  static_cast<cudaStream_t>(stream)));
}

size_t mikv_prefix_workspace_bytes(const mikv_prefix_desc* d) {
  if (prefix_ok(d) != MIKV_OK) return 0;
  return flash_workspace_bytes(d->groups, d->heads_kv, d->heads_q / d->heads_kv, d->batch / d->groups, d->length,
                               num_sms());
}

mikv_status mikv_prefix_attention(const mikv_prefix_desc* d, const void* q, const mikv_view* k, const mikv_view* v,
                                  const int32_t* lens, const int32_t* q_pos, const float* slopes,
                                  const float* own_out, const float* own_ml, void* out, float* ml, void* workspace,
                                  size_t ws_bytes, void* stream) {
  MIKV_CALL_RANGE();
  mikv_status st = prefix_ok(d);
  if (st != MIKV_OK) return st;
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !own_out != !own_ml) return MIKV_ERR_ARG;
  if (!aligned(lens, 4) || !aligned(q_pos, 4) || !aligned(slopes, 4) || !aligned(own_out, 16) || !aligned(own_ml, 8) ||
      !aligned(ml, 4))
    return MIKV_ERR_ARG;
  FlashArgs a;
  memset(&a, 0, sizeof a);
  const int per = d->batch / d->groups;
  long long s[3];
  if (d->length > 0) {
    if ((st = attn_view(k, d->groups, d->heads_kv, d->length, 2, true, s)) != MIKV_OK) return st;
    a.k = k->data, a.k_b = s[0], a.k_h = s[1], a.k_t = s[2];
    if ((st = attn_view(v, d->groups, d->heads_kv, d->length, 2, true, s)) != MIKV_OK) return st;
    a.v = v->data, a.v_b = s[0], a.v_h = s[1], a.v_t = s[2];
  }
  if (!workspace || !aligned(workspace, 256) || ws_bytes < mikv_prefix_workspace_bytes(d)) return MIKV_ERR_WORKSPACE;
  const long long row = (long long)d->heads_q * kHeadDim;
  a.q = q, a.q_b = per * row, a.q_h = kHeadDim, a.q_t = row;
  a.out = out, a.o_b = per * row, a.o_h = kHeadDim, a.o_t = row;
  a.stat = ml;
  a.stat_pair = 1;
  a.s_b = (long long)per * d->heads_q, a.s_h = 1, a.s_t = d->heads_q;
  a.own_out = own_out, a.own_ml = own_ml;
  a.lens = lens;
  a.pos = q_pos;
  a.pos_at_len = 1;
  a.slopes = slopes;
  a.batch = d->groups, a.tq = per, a.tk = d->length;
  a.heads_q = d->heads_q, a.heads_kv = d->heads_kv, a.G = d->heads_q / d->heads_kv;
  a.sm_scale = d->sm_scale, a.softcap = d->softcap;
  a.status = static_cast<int*>(workspace);
  return cuda_status(launch_flash(a, d->dtype == MIKV_F16, d->out_dtype == MIKV_F32, workspace, num_sms(),
                                  static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
