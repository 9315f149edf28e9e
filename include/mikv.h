/*
 * mikv.h — C ABI of libmikv: the GB300 (sm_103a) decode hot path of MiKV, the importance-aware
 * mixed-precision KV cache of "No Token Left Behind: Reliable KV Cache Compression via
 * Importance-Aware Mixed Precision Quantization" (arxiv 2402.18096).
 *
 * What the library computes, per attention layer and decode step:
 *   - important KV pairs (chosen by accumulated attention score, the heavy-hitter policy the paper
 *     plugs in, Fig. 4 / Sec. 3) stay in bf16 in the "important set";
 *   - all other KV pairs are kept, not evicted, as N-bit (N = 2, 3, 4) per-token group-wise asymmetric
 *     round-to-nearest codes with fp16 scale/zero (Eq. 1, Sec. 3.1) in the "retained set";
 *   - keys are multiplied by a per-channel balancer before quantization and the query is divided by
 *     it (Eq. 2-4, Sec. 3.2);
 *   - attention treats the two sets as one unordered set (permutation invariance, Sec. 3.4);
 *   - optionally (Sec. 3.3, Table 3) the important set itself is kept at reduced precision: INT8,
 *     INT4 or INT2 codes with fp16 scale/zero per 64 channels, quantized like the retained set.
 *
 * Conventions shared by every entry point:
 *   - All array pointers are DEVICE pointers owned by the caller; the library never allocates,
 *     frees or synchronises. Every call enqueues its kernels on `stream` (a cudaStream_t passed as
 *     void*, NULL = legacy default stream) and returns before they run.
 *   - Arguments are validated on the host before anything is launched; a call that returns an error
 *     has launched nothing (MIKV_ERR_CUDA excepted: a launch was attempted and failed).
 *   - bf16 = IEEE bfloat16, fp16 = IEEE binary16, both stored as 2-byte little-endian values.
 *   - Layouts are dense row-major in the index order written next to each argument.
 *   - The head dimension d is 128; the query-head group size G = heads_q / heads_kv is 1, 2, 4 or 8
 *     (grouped-query attention: query head j reads KV head j / G).
 *   - Each compute entry point (balancer, quantize/pack, prefill scores, attention, importance update,
 *     select/demote, insert, gather, decode step) marks its host time with one NVTX range named after
 *     the call (NVTX v3, header-only: inert unless a tool such as Nsight is attached; a build with
 *     -DMIKV_NVTX=0 leaves the ranges out).
 *
 * Packed-code layout of one retained row (d = 128, N bits, 16 * N bytes): channel c is written
 * c = 16 m + u (u = c mod 16, m = c div 16) and a plane is a sequence of little-endian 16-bit units.
 * In a plane of f-bit fields (f in {2, 4, 8}) with P = 16 / f codes per unit, channel c sits in unit
 * 8 * (2 * (m div P) + (u div 8)) + (u mod 8) at bits [f * (m mod P), f * (m mod P) + f). In a plane of
 * 1-bit fields, channel c sits in unit (u mod 8) at bit 2 * m + (u div 8). N = 2, 4 and 8 use one
 * plane of N-bit fields; N = 3 uses a plane of 2-bit fields (code bits 0..1) followed by a plane of
 * 1-bit fields (code bit 2). The quantization parameters of a row are d / group pairs of fp16
 * (alpha, beta), alpha first; the dequantized value is alpha * code + beta.
 */
#ifndef MIKV_H
#define MIKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MIKV_OK = 0,
  MIKV_ERR_ARG = 1,         /* null pointer, negative or inconsistent size */
  MIKV_ERR_UNSUPPORTED = 2, /* valid but not built: d != 128, bits not in {2,3,4}, ... */
  MIKV_ERR_CAPACITY = 3,    /* a write would pass lo_cap / hi_cap */
  MIKV_ERR_CUDA = 4,        /* a CUDA call failed; cudaGetLastError() was consumed */
  MIKV_ERR_WORKSPACE = 5,   /* workspace missing, too small or misaligned */
  MIKV_ERR_DEVICE = 6,      /* a kernel reported a failure through the workspace status word */
  MIKV_ERR_SCRATCH = 7      /* the problem needs more scratch than mikv_decode_attention_noalloc's
                               built-in buffer holds (MIKV_NOALLOC_SCRATCH_BYTES) */
} mikv_status;

/* Shape of one layer's mixed-precision cache. */
typedef struct {
  int32_t batch;     /* B */
  int32_t heads_q;   /* Hq, query heads */
  int32_t heads_kv;  /* Hkv, KV heads; Hq / Hkv in {1, 2, 4, 8} */
  int32_t head_dim;  /* d, must be 128 */
  int32_t bits;      /* N, retained-set code width: 2, 3 or 4 (Eq. 1); 0 = no retained set: demoted
                        tokens are evicted (the importance-based eviction baseline, H2O, Sec. 2.2 /
                        Fig. 2); the retained arrays are then unused and may be NULL, n_lo must be 0 */
  int32_t group;     /* g, channels per quantization group: 32, 64 or 128 (Sec. 3.2 uses d/2); ignored when bits = 0 */
  int32_t hi_cap;    /* important slots attended per head: the budget k plus one staging slot */
  int32_t hi_stride; /* rows per head in the important-set arrays: multiple of 16, >= hi_cap */
  int32_t lo_cap;    /* rows per head in the retained-set arrays: multiple of 16 */
  int32_t hi_bits;   /* important-set precision: 0 or 16 = bf16; 8, 4 or 2 = codes (Sec. 3.3, Table 3) */
  int32_t hi_group;  /* channels per group of a coded important set: 64 (ignored for bf16) */
  int32_t k_channel_group; /* 0: retained keys per token (Eq. 1, groups of `group` channels, balanced).
                              64: retained keys per CHANNEL over groups of 64 consecutive retained tokens
                              (App. C): one fp16 (alpha, beta) per (token group, channel), no balancer;
                              values stay per token. Retained tokens wait in bf16 in staging rows
                              hi_cap .. hi_cap + 63 of the important arrays until their group of 64 is
                              complete: of n_lo retained tokens, n_lo mod 64 are staged (in order) and
                              the rest quantized. Requires a bf16 important set, hi_stride >= hi_cap + 64
                              and lo_cap % 64 == 0; k_params is then fp16 [B][Hkv][lo_cap / 64][d][2]. */
} mikv_shape;

/* Device arrays of one layer's cache. Rows >= hi_cap of the important arrays are padding and are
 * never read as data; retained rows >= the current length likewise. */
typedef struct {
  void* k_hi;           /* bf16 [B][Hkv][hi_stride][d], keys WITHOUT the balancer; or, for a coded
                           important set, uint8 [B][Hkv][hi_stride][16 * hi_bits] codes of BALANCED keys */
  void* v_hi;           /* bf16 [B][Hkv][hi_stride][d]; or uint8 [B][Hkv][hi_stride][16 * hi_bits] */
  int32_t* hi_tok;      /* int32 [B][Hkv][hi_stride], token position held by each slot */
  float* acc;           /* fp32 [B][Hkv][hi_stride], accumulated attention score per slot */
  void* k_codes;        /* uint8 [B][Hkv][lo_cap][16 * bits], codes of balanced keys (Eq. 3) */
  void* v_codes;        /* uint8 [B][Hkv][lo_cap][16 * bits] */
  void* k_params;       /* fp16 [B][Hkv][lo_cap][d / group][2] (alpha, beta) */
  void* v_params;       /* fp16 [B][Hkv][lo_cap][d / group][2] */
  int32_t* lo_tok;      /* int32 [B][Hkv][lo_cap], token position of each retained row */
  const float* balancer; /* fp32 [Hkv][d] channel balancer of this layer (Eq. 2), or NULL = 1 */
  void* k_hi_params;    /* coded important set only (else unused): fp16 [B][Hkv][hi_stride][d / hi_group][2] */
  void* v_hi_params;    /* coded important set only: fp16 [B][Hkv][hi_stride][d / hi_group][2] */
} mikv_cache;

/* Output element type of mikv_decode_attention. */
enum { MIKV_OUT_BF16 = 0, MIKV_OUT_F32 = 1 };

/* Which operation a workspace is sized for (mikv_workspace_bytes). */
enum { MIKV_WS_ATTENTION = 0, MIKV_WS_BALANCER = 1, MIKV_WS_STEP = 2, MIKV_WS_PREFILL = 3 };

/* Human-readable name of a status code (static string). */
const char* mikv_status_string(mikv_status s);

/* Bytes of workspace `op` needs for `shape` with up to `n_lo_max` retained rows per head (the
 * attention split count depends on it; for MIKV_WS_PREFILL the third argument is the prefill length T). Returns 0 for an invalid shape. The workspace must be
 * 256-byte aligned; its first 16 bytes hold a status word that kernels set on an internal failure. */
size_t mikv_workspace_bytes(const mikv_shape* shape, int32_t op, int32_t n_lo_max);

/* Zero the workspace status word (enqueued on `stream`). */
mikv_status mikv_workspace_reset(void* workspace, size_t ws_bytes, void* stream);

/* Synchronise `stream`, read the workspace status word and return MIKV_ERR_DEVICE if a kernel
 * reported a failure (a wait that ran out of its iteration limit), else MIKV_OK. */
mikv_status mikv_workspace_check(const void* workspace, void* stream);

/*
 * Channel balancer, Eq. 2 (Sec. 3.2): balancer[h][c] = sqrt(max |q_pre| / max |k_pre|), the maxima
 * taken over all batch rows b, prefill tokens t < T and, for the query, the G query heads of KV head h
 * (the balanced keys are shared by those heads). A zero maximum on either side gives 1. fp32 IEEE
 * division and square root (bit-exact with a correctly rounded CPU evaluation).
 *   q_pre   bf16 [B][Hq][T][d] prefill queries (after positional embedding)
 *   k_pre   bf16 [B][Hkv][T][d] prefill keys
 *   balancer_out fp32 [Hkv][d]
 *   workspace >= mikv_workspace_bytes(shape, MIKV_WS_BALANCER, 0)
 */
mikv_status mikv_compute_balancer(const mikv_shape* shape, const void* q_pre, const void* k_pre,
                                  int32_t T, float* balancer_out, void* workspace, size_t ws_bytes,
                                  void* stream);

/*
 * Demotion into the retained set: Eq. 1 quantizer with Eq. 3 key balancing, group-wise per token.
 * For every (b, h) and i < n_rows, source row r = rows[b][h][i] (0 <= r < n_src) is quantized and
 * written to retained row lo_start + i:
 *   keys   x = bf16(k_src[b][h][r][c]) * balancer[h][c]  (fp32 product; balancer NULL => x = k)
 *   values x = bf16(v_src[b][h][r][c])
 *   per group of `group` channels: beta16 = fp16 rounded toward -inf of min(x); alpha16 = fp16 rounded
 *   toward +inf of fp32((max(x) - beta16) / (2^N - 1)) (1.0 when max(x) == beta16); code = clamp(
 *   round-half-even(fp32((x - beta16) / alpha16)), 0, 2^N - 1). Codes are packed as in the header.
 *   lo_tok[b][h][lo_start + i] = src_tok ? src_tok[b][h][r] : r.
 *   k_src, v_src  bf16 [B][Hkv][n_src][d], 16-byte aligned (e.g. the important arrays, n_src = hi_stride)
 *   src_tok       int32 [B][Hkv][n_src] or NULL
 *   rows          int32 [B][Hkv][n_rows]   (device; e.g. the output of mikv_select_demote)
 * Errors: MIKV_ERR_ARG if k_src or v_src is not 16-byte aligned; MIKV_ERR_CAPACITY if lo_start + n_rows >
 * lo_cap. Rows outside [0, n_src) are skipped by the kernel. Codes and parameters are bit-exact with an IEEE fp32 evaluation of the formulas above.
 */
/* With per-channel keys (k_channel_group = 64), mikv_quantize_pack APPENDS the rows at retained positions
 * lo_start .. lo_start + n_rows - 1, lo_start being the current retained length: a position whose group of
 * 64 completes is quantized with its group (keys per channel from the staged rows and the new ones, values
 * per token), the others are copied into the staging rows (bf16, keys unbalanced) with their token ids. */
mikv_status mikv_quantize_pack(const mikv_shape* shape, const mikv_cache* cache, const void* k_src,
                               const void* v_src, const int32_t* src_tok, int32_t n_src,
                               const int32_t* rows, int32_t n_rows, int32_t lo_start, void* stream);

/*
 * Initial importance of the prefill tokens: the accumulated attention each key receives from the prefill's
 * causal attention (the heavy-hitter score of Fig. 4 / Sec. 3, here taken over the prefill queries):
 *   scores[b][h][t] = sum over the G query heads j of KV head h and the queries i >= t of
 *                     exp(s_it - m_i) / l_i,  s_it = sm_scale * q_pre[b][hG+j][i] . k_pre[b][h][t],
 *   m_i = max_{t' <= i} s_it', l_i = sum_{t' <= i} exp(s_it' - m_i)  (the causal softmax of row i).
 * These are the scores mikv_select_demote / mikv_gather_hi take to build the cache. Two tensor-core
 * passes over the causal triangle (row statistics, then column sums), fp32 accumulation.
 *   q_pre      bf16 [B][Hq][T][d], 16-byte aligned (prefill queries after the positional embedding)
 *   k_pre      bf16 [B][Hkv][T][d], 16-byte aligned
 *   scores     fp32 [B][Hkv][T]
 *   workspace  >= mikv_workspace_bytes(shape, MIKV_WS_PREFILL, T) bytes, 256-byte aligned (the row
 *              statistics; its status word reports an internal failure as in the other entry points)
 * Only batch, heads_q, heads_kv and head_dim of `shape` are used. Requires B * Hq * T < 2^31.
 */
mikv_status mikv_prefill_scores(const mikv_shape* shape, const void* q_pre, const void* k_pre, int32_t T,
                                float sm_scale, float* scores, void* workspace, size_t ws_bytes, void* stream);

/*
 * The same sums where the queries attend to more than these keys (a prefix that requests share stands before them): the
 * weights are those of the whole softmax, whose log-sum-exp per query is given (mikv_prompt_attention's lse,
 * mikv_prefix_attention's ml):
 *   scores[b][h][t] = sum over the G query heads j of KV head h and the queries i >= t of exp(s_it - lse[b][hG+j][i])
 * A query whose lse is infinite weighs nothing. One tensor-core pass.
 *   lse        fp32 [B][Hq][T]
 *   the others as in mikv_prefill_scores
 */
mikv_status mikv_prefill_scores_lse(const mikv_shape* shape, const void* q_pre, const void* k_pre, int32_t T,
                                    float sm_scale, const float* lse, float* scores, void* workspace, size_t ws_bytes,
                                    void* stream);

/*
 * Single-token decode attention over the mixed-precision cache (Eq. 3-4; Sec. 3.4):
 *   s_i = sm_scale * q . k_hi[i]                  for the hi_cap important slots (bf16 keys)
 *   s_t = sm_scale * (q / balancer) . k_hat[t]    for retained rows t < n_lo, k_hat = alpha*code+beta
 *   out = sum_j softmax(s)_j * v_j  over both sets (v_hat = alpha * code + beta for retained rows)
 * A coded important set (hi_bits < 16) is attended like the retained set: s_i = sm_scale *
 * (q / balancer) . k_hat[i] with its own codes and parameters, values dequantized likewise.
 * Split-K flash decoding: partial (max, sum, unnormalised output) per context split in fp32, merged
 * into `out`. Arithmetic: fp32 accumulation; dot products on tensor cores with bf16 (important) or
 * fp16 (retained: dequantized codes, q / balancer) operands.
 *   q          bf16 [B][Hq][d]
 *   out        [B][Hq][d], bf16 (out_dtype MIKV_OUT_BF16) or fp32 (MIKV_OUT_F32)
 *   hi_logits  fp32 [B][Hq][hi_stride] or NULL: s_i of every important slot i < hi_cap
 *   ml         fp32 [B][Hq][2] or NULL: (m = max_j s_j, l = sum_j exp(s_j - m))
 *   workspace  >= mikv_workspace_bytes(shape, MIKV_WS_ATTENTION, n_lo) bytes, 256-byte aligned
 * Requires hi_cap + n_lo >= 1, 0 <= n_lo <= lo_cap. Every important slot < hi_cap must hold a token.
 */
mikv_status mikv_decode_attention(const mikv_shape* shape, const mikv_cache* cache, int32_t n_lo,
                                  const void* q, float sm_scale, void* out, int32_t out_dtype,
                                  float* hi_logits, float* ml, void* workspace, size_t ws_bytes,
                                  void* stream);

/*
 * Accumulated-attention importance (heavy-hitter) update: for every (b, h) and slot i < hi_cap,
 *   acc[b][h][i] += sum over the G query heads j of KV head h of exp(s_ji - m_j) / l_j
 * with s from hi_logits and (m, l) from ml as written by mikv_decode_attention. fp32.
 * Retained tokens are not tracked: once demoted a token cannot return to high precision.
 */
mikv_status mikv_update_importance(const mikv_shape* shape, const mikv_cache* cache,
                                   const float* hi_logits, const float* ml, void* stream);

/*
 * Demotion choice: per (b, h), the n_demote least important of n entries, ordered by
 * (score ascending, id ascending) — ties on the score demote the older token first.
 *   scores   fp32 [batch][heads][stride] (entries 0..n-1 are read; e.g. cache->acc with
 *            n = hi_cap and stride = hi_stride); scores must not be NaN
 *   ids      int32 [batch][heads][stride] or NULL (id = entry index); ids must be distinct per head
 *   demoted  int32 [batch][heads][n_demote]: entry indices of the demoted set, ascending
 *   kept     int32 [batch][heads][n - n_demote] or NULL: the remaining entries, ascending
 * Bit-exact: the selected set is fully determined by the order above.
 */
mikv_status mikv_select_demote(int32_t batch, int32_t heads, const float* scores,
                               const int32_t* ids, int32_t n, int32_t stride, int32_t n_demote,
                               int32_t* demoted, int32_t* kept, void* stream);

/*
 * New-token insertion (Fig. 4: the new KV pair enters the important set in high precision):
 * slot s = slots[b][h] (0 <= s < hi_cap) of every (b, h) receives k_new[b][h], v_new[b][h]
 * (bf16 [B][Hkv][d], keys without balancer), hi_tok = tok and acc = 0. With a coded important set
 * (hi_bits < 16) the rows are quantized on the way in (Eq. 1 at hi_bits, groups of hi_group; the key
 * multiplied by the balancer first, Eq. 3), exactly as mikv_quantize_pack quantizes retained rows.
 */
mikv_status mikv_insert_token(const mikv_shape* shape, const mikv_cache* cache, const void* k_new,
                              const void* v_new, int32_t tok, const int32_t* slots, void* stream);

/*
 * Important-set build from prefill rows: important slot i < n_rows of (b, h) receives source row
 * r = rows[b][h][i] of k_src/v_src (bf16 [B][Hkv][n_src][d]), hi_tok = src_tok ? src_tok[b][h][r] : r
 * and acc = src_scores ? src_scores[b][h][r] : 0. Requires n_rows <= hi_cap. A coded important set
 * receives the quantized rows (as in mikv_insert_token).
 */
mikv_status mikv_gather_hi(const mikv_shape* shape, const mikv_cache* cache, const void* k_src,
                           const void* v_src, const int32_t* src_tok, const float* src_scores,
                           int32_t n_src, const int32_t* rows, int32_t n_rows, void* stream);

/*
 * One whole decode step of one layer, in order: insert the new token into slots[b][h]
 * (mikv_insert_token), attend (mikv_decode_attention over hi_cap slots and n_lo retained rows),
 * update the importance scores (mikv_update_importance), choose the least important slot
 * (mikv_select_demote, n_demote = 1) and demote it to retained row n_lo (mikv_quantize_pack).
 * On return slots[b][h] holds the slot freed by the demotion (the next step's insertion slot);
 * the retained length becomes n_lo + 1. With bits = 0 (eviction) nothing is demoted: the victim's slot
 * is freed and the retained length stays 0. A coded important slot is demoted from its dequantized values:
 * per channel the fp32 value alpha * code + beta (rounded once), quantized at bits / group; keys are
 * already balanced and are not multiplied by the balancer again (Sec. 3.3).
 *   q, k_new, v_new   bf16 [B][Hq][d], [B][Hkv][d], [B][Hkv][d]
 *   slots             int32 [B][Hkv], in/out
 *   out               as in mikv_decode_attention
 *   workspace         >= mikv_workspace_bytes(shape, MIKV_WS_STEP, n_lo)
 * Errors: MIKV_ERR_CAPACITY if n_lo + 1 > lo_cap.
 */
mikv_status mikv_decode_step(const mikv_shape* shape, const mikv_cache* cache, int32_t n_lo,
                             const void* q, const void* k_new, const void* v_new, int32_t tok,
                             int32_t* slots, float sm_scale, void* out, int32_t out_dtype,
                             void* workspace, size_t ws_bytes, void* stream);

/*
 * Decode attention without a caller-provided workspace and without any allocation (there is no
 * counterpart in the paper; this is a deployment convenience).
 *
 * Some callers cannot allocate device memory on the decode path: an inference engine that owns every
 * byte of device memory through its own pool and forbids plugins from calling the CUDA allocator, or a
 * latency-critical serving loop that must not call cudaMalloc (it can synchronise the device). This
 * entry point computes exactly what mikv_decode_attention computes, with the same arguments minus the
 * workspace, and keeps its split partials in a scratch buffer that the library itself declares as a
 * fixed-size device array of MIKV_NOALLOC_SCRATCH_BYTES bytes. Every GPU that loads the library holds
 * that buffer until the process exits.
 *   - Every call looks up the buffer's device address in the current context (cudaGetSymbolAddress,
 *     which allocates nothing). The first call on a device (in a context) also loads the library's device
 *     code there: make that first call before any stream capture.
 *   - The call itself allocates nothing and frees nothing; it zeroes the buffer's status word on
 *     `stream` before launching.
 *   - All calls share the one buffer, which keeps the last call's contents: calls that can overlap on
 *     the GPU (different streams without ordering between them) race on it and must not be issued.
 *   - A problem whose scratch (mikv_workspace_bytes(shape, MIKV_WS_ATTENTION, n_lo)) exceeds the
 *     buffer returns MIKV_ERR_SCRATCH and launches nothing.
 *   - A kernel-side failure (a wait that ran out of its time limit) is recorded in the buffer's status
 *     word, not in the return code (the call returns before the kernels run): mikv_noalloc_check reads it.
 */
#define MIKV_NOALLOC_SCRATCH_BYTES (8u << 20)
mikv_status mikv_decode_attention_noalloc(const mikv_shape* shape, const mikv_cache* cache, int32_t n_lo,
                                          const void* q, float sm_scale, void* out, int32_t out_dtype,
                                          float* hi_logits, float* ml, void* stream);

/* Status of the built-in buffer of mikv_decode_attention_noalloc: synchronises `stream`, reads the buffer's
 * status word (left by the last mikv_decode_attention_noalloc call, which zeroed it first) and returns
 * MIKV_ERR_DEVICE if a kernel reported a failure, else MIKV_OK. Allocates nothing. */
mikv_status mikv_noalloc_check(void* stream);

/*
 * Debug builds. Every kernel that takes an index from device memory (an insertion slot in `slots`, a source row in
 * `rows`, the victim of a step) skips the access when the index is out of range, without error. A library built
 * with -DMIKV_DEBUG also records each such skip, and the internal invariants of the attention work split, as a
 * failure: in the workspace status word for the entry points with a workspace (read by mikv_workspace_check), and
 * in a status word of its own for mikv_insert_token, mikv_gather_hi and mikv_quantize_pack. No kernel traps.
 *   mikv_debug_enabled  1 if this library was built with -DMIKV_DEBUG, else 0. Host-only.
 *   mikv_debug_check    synchronises `stream`, reads and clears the library's own status word and returns
 *                       MIKV_ERR_DEVICE if an index check failed since the last call, else MIKV_OK (always
 *                       MIKV_OK in release builds).
 */
int32_t mikv_debug_enabled(void);
mikv_status mikv_debug_check(void* stream);

/*
 * KV-cache size as a fraction of an all-fp16 cache (the "Cache size" columns of Tables 2-3): a ratio
 * `ratio` of tokens kept at hi_bits (16 = fp16; otherwise hi_bits-bit codes plus fp16 alpha/beta per
 * group) and the rest at `bits`-bit codes plus fp16 alpha/beta per `group` channels:
 *   ratio * (hi_bits >= 16 ? 1 : (hi_bits + 32/group) / 16) + (1 - ratio) * (bits + 32/group) / 16.
 * Host-only, pure.
 */
double mikv_cache_fraction(int32_t bits, int32_t group, double ratio, int32_t hi_bits);

/*
 * Important-set budget from the importance ratio (the "Importance ratio" column of Tables 1-3: the share
 * of tokens kept in high precision): k = floor(ratio * T + 0.5), the ratio times the context length
 * rounded half up, evaluated in IEEE double arithmetic. A cache built for context T keeps k important
 * tokens and attends hi_cap = k + 1 important slots (one staging slot receives each decoded token before
 * the step's demotion frees a slot again). Returns -1 for T < 0 or a ratio outside [0, 1] (NaN included).
 * Host-only, pure.
 */
int32_t mikv_budget(int32_t T, double ratio);

/* Bytes of one retained row (codes + parameters, K or V) and of one important row (K or V). */
size_t mikv_retained_row_bytes(int32_t bits, int32_t group, int32_t head_dim);

/* ------------------------------------------------------------------ prompts: positions, attention, shared prefixes
 *
 * What stands on either side of the mixed-precision cache: rotary positions for queries and keys, the attention of
 * a prompt's own tokens, and single-token attention over a prefix whose keys and values several requests share
 * (joined with what each request's own cache gave). The conventions are those of the entry points above. Tensors
 * are views with strides, so the token-major rows a projection leaves and the head-major rows the cache is built
 * from are taken alike. */

/* Element types of these entry points. */
enum { MIKV_BF16 = 0, MIKV_F16 = 1, MIKV_F32 = 2 };

/* A tensor [batch][heads][tokens][d] in device memory: element strides of its first three dimensions (the channels
 * are dense). The stride of a dimension of size 1 is not used. */
typedef struct {
  void* data;
  int64_t stride_batch, stride_head, stride_token;
} mikv_view;

/* Which channels of a head turn together: i and i + rot / 2, or 2 i and 2 i + 1 (i < rot / 2). */
enum { MIKV_ROTARY_HALF = 0, MIKV_ROTARY_INTERLEAVED = 1 };

typedef struct {
  int32_t dtype;      /* of both tensors: MIKV_BF16, MIKV_F16 or MIKV_F32 */
  int32_t batch;
  int32_t tokens;
  int32_t heads_q;    /* heads of the first tensor */
  int32_t heads_k;    /* heads of the second tensor, 0 = there is none */
  int32_t head_dim;   /* d, must be 128 */
  int32_t rot;        /* channels that turn, even, 2 <= rot <= d; the others are copied */
  int32_t layout;     /* MIKV_ROTARY_HALF or MIKV_ROTARY_INTERLEAVED */
  int32_t inverse;    /* 0: turn by the angle; 1: by minus the angle: the transposed map (turns stored keys back; it is
                         also the map of gradients) */
  float amplitude;    /* factor on the turned channels (1 unless long-context scaling asks for one) */
} mikv_rotary_desc;

/*
 * Phases of the rotary frequencies: phases[i] = the fraction of a turn that frequency i (radians per position,
 * freq[i] >= 0) advances per position, modulo 1, in units of 2^-64. Position times phase in 64-bit integer
 * arithmetic is then the angle modulo a turn, without the loss that a 32-bit product has at long positions.
 * Host-only, pure; n values each. Returns MIKV_ERR_ARG for a negative or non-finite frequency.
 */
mikv_status mikv_rotary_phases(const double* freq, int32_t n, uint64_t* phases);

/*
 * Rotary positions of a query tensor and (optionally, in the same launch) a key tensor: every pair (x, x') of
 * channels named by `layout` becomes amplitude * (x cos a - x' sin a, x sin a + x' cos a), a = 2 pi pos phase_i,
 * the other channels are copied; fp32 arithmetic, one rounding to `dtype`.
 *   q_in, q_out, k_in, k_out  views [batch][heads][tokens][d]; an output may be its own input (in place), and may
 *              have other strides than it (e.g. token-major in, head-major out). Any alignment of the elements.
 *   phases     uint64 [rot / 2] (device), see mikv_rotary_phases
 *   positions  int32 [batch][tokens] (device), or NULL: token t has position `start` + t. Negative positions turn
 *              the other way.
 * With no tokens nothing is launched and no view is looked at.
 */
mikv_status mikv_rotary(const mikv_rotary_desc* desc, const mikv_view* q_in, const mikv_view* q_out,
                        const mikv_view* k_in, const mikv_view* k_out, const uint64_t* phases,
                        const int32_t* positions, int32_t start, void* stream);

/*
 * The keys that each query of a prompt sees, as half-open spans: spans[b][i] = [lo, hi). Query i stands at position
 * p = q_start + i among the tk keys. It starts from [0, causal ? p + 1 : tk); then
 *   docs    int32 [batch][n_docs + 1] or NULL: ascending offsets of the documents packed into the row. lo becomes
 *           the start of the document that holds p, hi is cut at its end; a p in no document (padding) sees nothing
 *   prefix  int32 [batch][max(n_docs, 1)] or NULL: the first prefix[d] keys of p's document (of the row without
 *           `docs`) are seen by all of its queries
 *   key_len int32 [batch] or NULL: keys from key_len[b] on are seen by nobody
 * An empty span is written as [0, 0). One launch; the result serves every layer of the batch.
 *   spans   int32 [batch][tq][2] (device), 8-byte aligned; may be NULL with no queries
 */
mikv_status mikv_mask_spans(int32_t* spans, int32_t batch, int32_t tq, int32_t tk, int32_t q_start, int32_t causal,
                            const int32_t* docs, int32_t n_docs, const int32_t* prefix, const int32_t* key_len,
                            void* stream);

typedef struct {
  int32_t dtype;      /* of q, k, v: MIKV_BF16 or MIKV_F16 */
  int32_t out_dtype;  /* of out: the same, or MIKV_F32 */
  int32_t batch;
  int32_t heads_q;
  int32_t heads_kv;   /* heads_q / heads_kv in {1, 2, 4, 8} */
  int32_t head_dim;   /* d, must be 128 */
  int32_t tq;         /* queries per row of the batch */
  int32_t tk;         /* keys per row of the batch */
  int32_t causal;     /* without spans: 1 = query i sees the keys up to its own position, 0 = all keys */
  int32_t q_start;    /* position of query 0 among the keys (tk - tq when the queries are the last tokens); at most
                         2^30 either way */
  float sm_scale;     /* > 0 */
  float softcap;      /* 0 = none; c > 0: scores become c tanh(score / c) */
} mikv_prompt_desc;

/*
 * Attention of a prompt's queries over its keys:
 *   s_ij = sm_scale * q_i . k_j;  softcap c: s_ij = c tanh(s_ij / c);  slopes: s_ij -= slope_h |p_i - j|
 *   out_i = sum_j softmax_j(s_i) v_j over the keys j that query i sees,  lse_i = ln sum_j exp(s_ij)
 * with p_i = q_start + i. A query that sees no key gives out = 0 and lse = -inf. Keys that no query sees may hold
 * any bits. A query that sees an infinity or NaN in V gets an infinity or NaN in the channels concerned (in tiles of 128
 * keys that a mask cuts for it or for a query worked on with it, NaN in all channels; which of the two an infinity
 * gives depends on its weight and on the number of queries); other queries are not touched by it (beyond the rounding
 * of their own sums).
 * Scores and sums are fp32 (exact products, fp32 accumulation; the cap within 2^-20 of its size, distances exact to
 * 2^24); the probabilities enter the product with V rounded to the input type, whatever out_dtype is. Results do not
 * depend on what else runs, and repeat bit for bit.
 *   q, k, v, out  views; 16-byte aligned data, strides multiples of 16 bytes. k and v may have a zero batch or head
 *                 stride (one set of keys for several)
 *   spans     int32 [batch][tq][2] from mikv_mask_spans, or NULL (then `causal` decides); lo < 0 counts as 0 and
 *             hi > tk as tk
 *   slopes    fp32 [heads_q] or NULL
 *   lse       fp32 [batch][heads_q][tq] or NULL
 *   workspace >= mikv_prompt_workspace_bytes(desc) bytes, 256-byte aligned, status word as in the entry points above
 */
size_t mikv_prompt_workspace_bytes(const mikv_prompt_desc* desc);
mikv_status mikv_prompt_attention(const mikv_prompt_desc* desc, const mikv_view* q, const mikv_view* k,
                                  const mikv_view* v, const mikv_view* out, const int32_t* spans,
                                  const float* slopes, float* lse, void* workspace, size_t ws_bytes, void* stream);

typedef struct {
  int32_t dtype;      /* of q, k, v: MIKV_BF16 or MIKV_F16 */
  int32_t out_dtype;  /* of out: the same, or MIKV_F32 */
  int32_t batch;      /* requests, one query token each */
  int32_t groups;     /* prefixes; requests b of the batch share prefix b div (batch / groups) */
  int32_t heads_q;
  int32_t heads_kv;   /* heads_q / heads_kv in {1, 2, 4, 8} */
  int32_t head_dim;   /* d, must be 128 */
  int32_t length;     /* keys per prefix (the longest, with `lens`) */
  float sm_scale;     /* > 0 */
  float softcap;      /* as in mikv_prompt_desc */
} mikv_prefix_desc;

/*
 * Single-token attention over prefixes that requests share: every key and value of a prefix is read once for all
 * its requests and their query heads. groups = batch gives each request keys of its own (a plain bf16 / fp16
 * cache); groups = 1 one prefix for all. Scores as in mikv_prompt_attention with p = q_pos[b].
 * With own_out and own_ml the result is joined with attention over other keys of the same query, as
 * mikv_decode_attention leaves it for the request's own cache (fp32 output, (max, sum)): the softmax runs over both. Own
 * parts have to come from scores of the same form: mikv_decode_attention has neither cap nor bias, so with those the own
 * part is another call's (this one's, with groups = batch, over a 16-bit cache of the request).
 *   q         [batch][heads_q][d] dense, 16-byte aligned
 *   k, v      views [groups][heads_kv][length][d] as in mikv_prompt_attention
 *   lens      int32 [groups] (device) or NULL: keys of each prefix, 0 <= lens <= length; later rows may hold any bits
 *   q_pos     int32 [batch] (device) or NULL: position of each query, for the distance (NULL: the prefix's length)
 *   slopes    fp32 [heads_q] or NULL
 *   own_out   fp32 [batch][heads_q][d], own_ml fp32 [batch][heads_q][2], or both NULL
 *   out       [batch][heads_q][d] dense, 16-byte aligned; 0 where there is no key at all
 *   ml        fp32 [batch][heads_q][2] or NULL: (ln sum exp(s), 1) over all keys, (-inf, 0) where there is none: a
 *             (reference, sum) pair like mikv_decode_attention's, for mikv_update_importance or a further join
 *   workspace >= mikv_prefix_workspace_bytes(desc) bytes, 256-byte aligned
 */
size_t mikv_prefix_workspace_bytes(const mikv_prefix_desc* desc);
mikv_status mikv_prefix_attention(const mikv_prefix_desc* desc, const void* q, const mikv_view* k,
                                  const mikv_view* v, const int32_t* lens, const int32_t* q_pos,
                                  const float* slopes, const float* own_out, const float* own_ml, void* out,
                                  float* ml, void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MIKV_H */
