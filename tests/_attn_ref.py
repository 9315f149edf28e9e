"""Attention over 16-bit keys in 64 bits, from the definition, with bounds on what the kernels may be off by."""
from __future__ import annotations

import math

import torch

# unit roundoffs: the probabilities and the output are rounded to these types
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# 128 exact products accumulated in fp32 by the tensor cores: a few 2^-23 of the sum of magnitudes, with margin
ACC_GAMMA = 2.0 ** -19


def span_mask(lo, hi, tk):
    """bool [..., tk] from lo, hi [...]"""
    j = torch.arange(tk, device=lo.device)
    return (j >= lo[..., None]) & (j < hi[..., None])


def spans_brute(B, tq, tk, q_start, causal, docs=None, prefix=None, key_len=None):
    """[B][tq] (lo, hi) of the documented rules, in plain Python."""
    out = []
    for b in range(B):
        row = []
        for i in range(tq):
            p = q_start + i
            keys = set(range(tk))
            doc = 0
            start = 0
            if docs is not None:
                doc = next((d for d in range(len(docs[b]) - 1) if docs[b][d] <= p < docs[b][d + 1]), None)
                if doc is None:
                    row.append((0, 0))
                    continue
                start = docs[b][doc]
                keys &= set(range(docs[b][doc], docs[b][doc + 1]))
            n = 0
            if prefix is not None:
                n = prefix[b][doc] if docs is not None else prefix[b]
            if causal:
                keys = {j for j in keys if j <= p or j < start + n}
            if key_len is not None:
                keys = {j for j in keys if j < key_len[b]}
            row.append((min(keys), max(keys) + 1) if keys else (0, 0))
        out.append(row)
    return torch.tensor(out, dtype=torch.int32)


def attention(q, k, v, mask, scale, cap=0.0, slopes=None, pos=None, out_dtype=None):
    """q [R, d] rows, k, v [T, d], mask [R, T]; slopes, pos [R] or None. Returns (out, lse, out bound, lse bound) in
    64 bits. Masked keys do not enter at all (whatever they hold).

    The bounds follow the arithmetic: scores are exact products accumulated in fp32 (E0), the cap is evaluated with an
    error of 2^-20 of its size (it does not enlarge E0), the bias and scaling round once each; weights are then off by
    a factor e^(2 E) and 2^-20 for the exponential and the sum, and by one rounding to the input type; the output is
    rounded once. The fp16 weights also lose what lies 2^-33 below the row's largest."""
    qd = q.double()
    live = mask.any(dim=0)
    kd = torch.where(live[:, None], k.double(), 0.0)
    vd = torch.where(live[:, None], v.double(), 0.0)
    s = scale * (qd @ kd.T)
    E = scale * ACC_GAMMA * (qd.abs() @ kd.abs().T) + 2.0 ** -22 * s.abs()
    if cap:
        s = cap * torch.tanh(s / cap)
        E = E + 2.0 ** -20 * cap
    if slopes is not None:
        dist = (pos.double()[:, None] - torch.arange(k.shape[0], device=k.device)).abs()
        s = s - slopes.double()[:, None] * dist
        E = E + 2.0 ** -21 * slopes.double()[:, None] * dist
    s = s.masked_fill(~mask, -math.inf)
    lse = torch.logsumexp(s, dim=1)
    w = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    # keys that weigh nothing do not move the result, whatever their score's error
    Em = torch.where(w > 2.0 ** -60, E, 0.0).amax(dim=1)
    out = w @ vd
    u = UNIT[q.dtype]
    rel = u + torch.expm1(2 * Em) + 2.0 ** -19
    mag = w @ vd.abs()
    tail = (mask.sum(dim=1) * 2.0 ** -33)[:, None] * vd.abs().amax(dim=0) if q.dtype == torch.float16 else 0.0
    inner = 2 * rel[:, None] * mag + tail
    bound = inner + UNIT[out_dtype or q.dtype] * (out.abs() + inner)
    if (out_dtype or q.dtype) == torch.float16:
        bound = bound + 2.0 ** -25  # subnormal outputs
    return out, lse, bound, Em + 2.0 ** -19 + 2.0 ** -22 * torch.where(lse == -math.inf, 0.0, lse).abs()


def join(out, lse, bound, lse_bound, own_out, own_ml, out_dtype):
    """The softmax over both parts, and its bounds: the part's own bound, the weights of the parts (they move with
    lse), and the rounding of the joined output."""
    mine = own_ml[:, 0].double() + torch.log(own_ml[:, 1].double())
    both = torch.logaddexp(lse, mine)
    a, b = torch.exp(lse - both)[:, None], torch.exp(mine - both)[:, None]
    o = out * a + own_out.double() * b
    slack = (2 * lse_bound + 2.0 ** -19)[:, None] * (out.abs() * a + own_out.double().abs() * b)
    return o, both, bound + slack + UNIT[out_dtype] * o.abs(), lse_bound + 2.0 ** -20 + 2.0 ** -22 * both.abs()
