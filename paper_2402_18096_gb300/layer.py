"""Cache build and decode steps of one attention layer, as a sequence of libmikv calls.

This is the flow a serving stack runs around the library (Fig. 4 of arxiv 2402.18096):
  prefill  -> channel balancer from prefill maxima (Eq. 2)
           -> choose the k most important tokens by accumulated attention (mikv_select_demote)
           -> keep them in high precision (mikv_gather_hi: bf16, or 8/4/2-bit codes for a reduced-
              precision important set, Sec. 3.3), quantize the rest into the retained set
              (mikv_quantize_pack, Eq. 1 with Eq. 3 key balancing)
  decode   -> per token: insert, attend, update importance, demote the least important (mikv_decode_step)
Requests that share a long prompt prefix keep it once, in bf16, beside a mixed-precision cache of their own tokens
(SharedPrefixLayer): rotary positions, prompt attention, and decode steps whose attention joins both.
Every step runs in the library's kernels; this module only orders the calls and owns the buffers.
"""
from __future__ import annotations

import math

import torch

from . import (LayerCache, MikvError, RotaryTable, Shape, WS_ATTENTION, WS_BALANCER, WS_PREFILL, WS_STEP, mikv_compute_balancer,
               mikv_decode_attention, mikv_decode_step, mikv_gather_hi, mikv_insert_token,
               mikv_prefill_scores, mikv_prefix_attention, mikv_prefix_workspace_bytes, mikv_prompt_attention,
               mikv_prompt_workspace_bytes, mikv_quantize_pack, mikv_rotary, mikv_select_demote,
               mikv_update_importance, mikv_workspace_bytes, mikv_workspace_check)


def workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A 256-byte aligned uint8 device buffer of at least nbytes (torch allocations are aligned)."""
    return torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=device)


class MixedPrecisionLayer:
    """One layer's MiKV cache plus the per-step state (free slots, retained length, workspace)."""

    def __init__(self, shape: Shape, balancer: torch.Tensor = None, device="cuda"):
        self.shape = shape
        self.cache = LayerCache(shape, device=device, balancer=balancer)
        self.slots = torch.zeros(shape.batch, shape.heads_kv, dtype=torch.int32, device=device)
        self.ws = workspace(mikv_workspace_bytes(shape, WS_STEP, shape.lo_cap), device)
        self.n_lo = 0
        self.pos = 0
        self.sm_scale = 1.0 / math.sqrt(shape.head_dim)

    @classmethod
    def from_prefill(cls, shape: Shape, k, v, scores, q_pre=None, budget: int = None, device="cuda"):
        """Build the cache from prefill K, V [B, Hkv, T, d] (bf16) and importance scores [B, Hkv, T].
        With q_pre [B, Hq, T, d] the channel balancer is computed (Eq. 2; not for per-channel keys, which
        need none); without it, b = 1. With scores
        None the importance is the prefill's accumulated causal attention (mikv_prefill_scores, q_pre
        required)."""
        B, H, T, _ = k.shape
        if scores is None:
            if q_pre is None:
                raise ValueError("prefill scores need the prefill queries")
            scores = torch.empty(B, H, T, dtype=torch.float32, device=device)
            ws = workspace(mikv_workspace_bytes(shape, WS_PREFILL, T), device)
            mikv_prefill_scores(shape, q_pre, k, scores, ws)
        k_budget = shape.hi_cap - 1 if budget is None else budget
        bal = None
        if q_pre is not None and not shape.k_channel_group:
            bal = torch.empty(H, shape.head_dim, dtype=torch.float32, device=device)
            ws = workspace(mikv_workspace_bytes(shape, WS_BALANCER, 0), device)
            mikv_compute_balancer(shape, q_pre, k, bal, ws)
        layer = cls(shape, balancer=bal, device=device)
        n_demote = T - k_budget
        demoted = torch.empty(B, H, n_demote, dtype=torch.int32, device=device)
        kept = torch.empty(B, H, k_budget, dtype=torch.int32, device=device)
        mikv_select_demote(scores, T, n_demote, demoted, kept)
        if k_budget > 0:
            mikv_gather_hi(layer.cache, k, v, kept, src_scores=scores)
        if n_demote > 0 and shape.bits:
            mikv_quantize_pack(layer.cache, k, v, demoted, 0)
        layer.n_lo = n_demote if shape.bits else 0  # bits = 0: eviction, the demoted tokens are dropped
        layer.pos = T
        layer.slots.fill_(k_budget)  # the staging slot receives the first decoded token
        return layer

    def step(self, q, k_new, v_new, out):
        """One decode step: the new token enters, attention runs, the least important slot is demoted."""
        mikv_decode_step(self.cache, self.n_lo, q, k_new, v_new, self.pos, self.slots, self.sm_scale, out,
                         self.ws)
        if self.shape.bits:
            self.n_lo += 1
        self.pos += 1


class SharedPrefixLayer:
    """One layer for a batch of requests whose prompts begin with the same tokens. The prefix's keys and values stay in
    bf16 and are read once per step for all requests; every request's own tokens live in a mixed-precision cache
    (bf16 important set). Queries and keys come in as projected, without positions; tensors are [B, H, T, d] views."""

    def __init__(self, own: MixedPrecisionLayer, k_prefix, v_prefix, table: RotaryTable):
        s = own.shape
        if s.hi_coded:
            raise ValueError("SharedPrefixLayer: the important set of the own cache is bf16")
        dev = k_prefix.device
        self.own, self.table = own, table
        self.k_prefix, self.v_prefix = k_prefix, v_prefix  # [1, Hkv, P, d], positions applied
        self.prefix = k_prefix.shape[2]
        like = torch.empty(s.batch, s.heads_q, s.head_dim, dtype=torch.bfloat16, device=dev)
        f = dict(dtype=torch.float32, device=dev)
        self.own_out = torch.empty(s.batch, s.heads_q, s.head_dim, **f)
        self.own_ml = torch.empty(s.batch, s.heads_q, 2, **f)
        self.ml = torch.empty(s.batch, s.heads_q, 2, **f)
        self.logits = torch.empty(s.batch, s.heads_q, s.hi_stride, **f)
        self.demoted = torch.empty(s.batch, s.heads_kv, 1, dtype=torch.int32, device=dev)
        self.ws_own = workspace(mikv_workspace_bytes(s, WS_ATTENTION, s.lo_cap), dev)
        self.ws_prefix = workspace(mikv_prefix_workspace_bytes(like, k_prefix), dev)
        self.prompt_status = None  # the status words that the prompts' calls left (from_prompts)

    @classmethod
    def from_prompts(cls, shape: Shape, table: RotaryTable, prefix, own, out_prefix, out_own, key_len=None):
        """The prompts of a batch: prefix = (q, k, v) of the shared tokens ([1, H, P, d], bf16), own = (q, k, v) of each
        request's own tokens ([B, H, T, d]). Turns q and k (in place), attends the prefix (into out_prefix) and the
        own tokens over prefix and own keys (into out_own), and builds the own cache by accumulated attention: the
        weights of the softmax over prefix and own keys, as in step. shape is the own cache's (shape_for_context with
        context = T).
        Every request has all T own tokens: key_len is refused. The cache holds the same number of slots and rows for
        every request and its attention weighs all of them, so the padding of a shorter one would be kept, attended and
        counted, and its next token would stand at a wrong position. Requests of other lengths go into other layers."""
        if key_len is not None:
            raise ValueError("SharedPrefixLayer: key_len (own tokens of several lengths) is not supported by the own cache")
        q0, k0, v0 = prefix
        q, k, v = own
        B, Hkv, T, d = k.shape
        Hq, P, dev = q.shape[1], k0.shape[2], k.device
        mikv_rotary(table, q0, k0)
        mikv_rotary(table, q, k, start=P)
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        rows = q.transpose(1, 2).contiguous().view(B * T, Hq, d)  # every own token a request of the prefix
        ws = workspace(max(mikv_prompt_workspace_bytes(q0, k0), mikv_prompt_workspace_bytes(q, k),
                           mikv_prefix_workspace_bytes(rows, k0), mikv_workspace_bytes(shape, WS_PREFILL, T)), dev)
        if P > 0:
            mikv_prompt_attention(q0, k0, v0, out_prefix, ws)
        # the own tokens over their own keys, joined with their attention over the prefix as it lies
        own_out = torch.empty(B, T, Hq, d, dtype=torch.float32, device=dev)
        lse = torch.empty(B, Hq, T, dtype=torch.float32, device=dev)
        mikv_prompt_attention(q, k, v, own_out.transpose(1, 2), ws, lse=lse)
        own_ml = torch.stack([lse, torch.ones_like(lse)], dim=3).transpose(1, 2).reshape(B * T, Hq, 2)
        ml = torch.empty_like(own_ml)
        joined = out_own.transpose(1, 2)
        if not joined.is_contiguous():
            joined = torch.empty(B, T, Hq, d, dtype=out_own.dtype, device=dev)
        mikv_prefix_attention(rows, k0, v0, joined.view(B * T, Hq, d), ws, own_out=own_out.view(B * T, Hq, d),
                              own_ml=own_ml, ml=ml)
        if joined.data_ptr() != out_own.data_ptr():
            out_own.copy_(joined.transpose(1, 2))
        lse.copy_(ml[:, :, 0].view(B, T, Hq).transpose(1, 2))
        del rows, own_out, own_ml, joined
        scores = torch.empty(B, Hkv, T, dtype=torch.float32, device=dev)
        mikv_prefill_scores(shape, q, k, scores, ws, lse=lse)
        layer = MixedPrecisionLayer.from_prefill(shape, k, v, scores, q, device=dev)
        layer = cls(layer, k0.contiguous(), v0.contiguous(), table)
        layer.prompt_status = ws[:256].clone()  # (the workspace itself is not kept)
        return layer

    def check(self, stream=None):
        """Raise MikvError (MIKV_ERR_DEVICE) if a kernel of the prompts or of a step so far gave up; synchronises."""
        for ws in (self.prompt_status, self.ws_prefix, self.ws_own):
            if ws is not None:
                mikv_workspace_check(ws, stream)

    def step(self, q, k_new, v_new, out):
        """One decode step: q [B, Hq, d], k_new, v_new [B, Hkv, d] of the new token as projected (q and k_new are turned
        in place) into out [B, Hq, d] (bf16 or fp32). The importance update takes the weights of the softmax over both
        parts. A call that is refused has changed nothing."""
        o, c = self.own, self.own.cache
        s = o.shape
        for name, t, heads, types in (("q", q, s.heads_q, (torch.bfloat16,)), ("k_new", k_new, s.heads_kv, (torch.bfloat16,)),
                                      ("v_new", v_new, s.heads_kv, (torch.bfloat16,)),
                                      ("out", out, s.heads_q, (torch.bfloat16, torch.float32))):
            if t.shape != (s.batch, heads, s.head_dim) or t.dtype not in types or not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"{name}: expected a dense device tensor of shape {(s.batch, heads, s.head_dim)} and type "
                                 f"{' or '.join(str(x) for x in types)}, got {t.dtype} {tuple(t.shape)}")
        if s.bits and o.n_lo >= s.lo_cap:
            raise MikvError("SharedPrefixLayer.step", 3)  # MIKV_ERR_CAPACITY: no row is left for the demoted token
        mikv_rotary(self.table, q[:, :, None], k_new[:, :, None], start=self.prefix + o.pos)
        mikv_insert_token(c, k_new, v_new, o.pos, o.slots)
        mikv_decode_attention(c, o.n_lo, q, o.sm_scale, self.own_out, self.ws_own, hi_logits=self.logits, ml=self.own_ml)
        mikv_prefix_attention(q, self.k_prefix, self.v_prefix, out, self.ws_prefix, own_out=self.own_out,
                              own_ml=self.own_ml, ml=self.ml)
        mikv_update_importance(c, self.logits, self.ml)
        mikv_select_demote(c.acc, s.hi_cap, 1, self.demoted, ids=c.hi_tok)
        if s.bits:
            mikv_quantize_pack(c, c.k_hi, c.v_hi, self.demoted, o.n_lo, src_tok=c.hi_tok)
            o.n_lo += 1
        o.slots.copy_(self.demoted[:, :, 0])
        o.pos += 1


def oracle_eviction_attention(k, v, q, budget: int, sm_scale: float, out, device="cuda"):
    """Oracle eviction (Sec. 2.2, Fig. 2), the comparison baseline: attention computed over the full bf16
    cache k, v [B, Hkv, T, d] for q [B, Hq, d], then top-k sparsity imposed on the attention map. Reading:
    each query head keeps its `budget` largest attention weights (ties: the smaller token index) and the
    output is the softmax over the logits of those tokens (the kept weights renormalised). Built from the
    library's entry points only: full attention with its logits, selection of the T - budget smallest
    logits (mikv_select_demote) whose complement is kept, gather of the kept rows, and attention over them; query heads of a KV head are handled one by one
    because each keeps its own tokens. Writes out [B, Hq, d]; returns the kept token indices [B, Hq, budget]."""
    B, H, T, d = k.shape
    Hq = q.shape[1]
    G = Hq // H
    full = Shape(B, H, H, 2, 32, T, 16)  # one query head per KV head at a time; bf16 important set of T rows
    cache = LayerCache(full, device=device)
    rows = torch.arange(T, dtype=torch.int32, device=device).expand(B, H, T).contiguous()
    mikv_gather_hi(cache, k, v, rows)
    kept_all = torch.empty(B, Hq, budget, dtype=torch.int32, device=device)
    small = Shape(B, H, H, 2, 32, budget, 16)
    ws = workspace(max(mikv_workspace_bytes(full, 0, 0), mikv_workspace_bytes(small, 0, 0)), device)
    # ids T-1-t: among equal logits the larger token index is dropped first, so the smaller one is kept
    ids = torch.arange(T - 1, -1, -1, dtype=torch.int32, device=device).expand(B, H, T).contiguous()
    ids = torch.nn.functional.pad(ids, (0, full.hi_stride - T))
    for j in range(G):
        qj = q[:, j::G].contiguous()
        logits = torch.empty(B, H, full.hi_stride, dtype=torch.float32, device=device)
        tmp = torch.empty(B, H, d, dtype=torch.float32, device=device)
        mikv_decode_attention(cache, 0, qj, sm_scale, tmp, ws, hi_logits=logits)
        kept = torch.empty(B, H, budget, dtype=torch.int32, device=device)
        dropped = torch.empty(B, H, T - budget, dtype=torch.int32, device=device)
        mikv_select_demote(logits, T, T - budget, dropped, kept=kept, ids=ids)
        sel = LayerCache(small, device=device)
        mikv_gather_hi(sel, k, v, kept)
        oj = torch.empty(B, H, d, dtype=out.dtype, device=device)
        mikv_decode_attention(sel, 0, qj, sm_scale, oj, ws)
        out[:, j::G] = oj
        kept_all[:, j::G] = kept
    return kept_all
