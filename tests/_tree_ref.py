"""Drafted tokens over a mixed-precision cache in 64 bits, from the definitions, with bounds on what the kernels may be
off by; caches of any bits to run them on."""
from __future__ import annotations

import math

import torch

import paper_2402_18096_gb300 as pkg

ACC_GAMMA = 2.0 ** -19  # a few 2^-23 of the sum of magnitudes of 128 products summed in fp32 by the tensor cores
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U16 = 2.0 ** -11


def gen(seed, device="cuda"):
    return torch.Generator(device=device).manual_seed(seed)


def codes_of(packed, bits):
    """int64 [..., 128] codes of packed rows, channel by channel from the layout's words."""
    w = packed.to(torch.int64)
    w = w[..., 0::2] | (w[..., 1::2] << 8)
    f = 2 if bits == 3 else bits
    P = 16 // f
    out = []
    for c in range(128):
        m, u = c // 16, c % 16
        x = (w[..., 8 * (2 * (m // P) + u // 8) + u % 8] >> (f * (m % P))) & ((1 << f) - 1)
        if bits == 3:
            x = x | (((w[..., 16 + u % 8] >> (2 * m + u // 8)) & 1) << 2)
        out.append(x)
    return torch.stack(out, dim=-1)


def values_of(packed, params, bits):
    p = params.double()
    g = 128 // p.shape[-2]
    return p[..., 0].repeat_interleave(g, -1) * codes_of(packed, bits) + p[..., 1].repeat_interleave(g, -1)


class Drafts:
    """A cache with random contents, drafted tokens for it, and what the requests hold. Slots and rows that are not in
    use, the free slots and padding nodes hold NaN (codes: any bits, NaN parameters). `tokens`: the cache's size at least,
    over all KV heads; rows behind lo_cap are there but not in use."""

    tokens = 0

    def __init__(self, seed, B, Hq, Hkv, nodes, hi_cap, lo_cap, bits=2, group=32, n_hi=None, n_lo=None, free=True,
                 balanced=True, parents=None, outliers=3.0, major=True):
        g = gen(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        rows = max(lo_cap, -(-self.tokens // (16 * B * Hkv)) * 16)
        self.shape = s = pkg.Shape(B, Hq, Hkv, bits, group, hi_cap, rows)
        self.cache = c = pkg.LayerCache(s)
        self.N, self.G = nodes, Hq // Hkv
        n_hi = [hi_cap] * B if n_hi is None else n_hi
        n_lo = [lo_cap if bits else 0] * B if n_lo is None else n_lo
        self.n_hi, self.n_lo = n_hi, n_lo
        c.balancer = torch.exp(0.7 * r(Hkv, 128)) if balanced else None
        c.k_hi.copy_(r(B, Hkv, s.hi_stride, 128)), c.v_hi.copy_(r(B, Hkv, s.hi_stride, 128))
        c.k_hi[..., 5] *= outliers
        c.k_hi[..., 69] *= outliers
        c.acc.copy_(torch.exp(r(B, Hkv, s.hi_stride)))
        c.hi_tok.copy_(torch.rand(B, Hkv, s.hi_stride, generator=g, device="cuda").argsort(2))
        for x in (c.k_codes, c.v_codes):
            x.copy_(torch.randint(0, 256, x.shape, generator=g, device="cuda"))
        if bits:
            for x, bal in ((c.k_params, c.balancer), (c.v_params, None)):
                span = 2.0 + 3.0 * torch.rand(*x.shape[:-1], generator=g, device="cuda")
                if bal is not None:  # groups of balanced keys: about the balancer's size
                    span = span * bal.view(Hkv, 1, -1, group).amax(-1).expand(B, Hkv, 1, -1).expand(span.shape)
                x[..., 0] = span / (2 ** bits - 1)
                x[..., 1] = -span * (0.3 + 0.4 * torch.rand(*x.shape[:-1], generator=g, device="cuda"))
        self.free = None
        if free:
            self.free = torch.tensor([[int(x) for x in torch.randint(0, max(n, 1), (Hkv,), generator=g, device="cuda")]
                                      for n in n_hi], dtype=torch.int32, device="cuda").view(B, Hkv)
        nan = math.nan
        for b in range(B):
            c.k_hi[b, :, n_hi[b]:], c.v_hi[b, :, n_hi[b]:] = nan, nan
            c.k_params[b, :, n_lo[b]:], c.v_params[b, :, n_lo[b]:] = nan, nan
            for h in range(Hkv):
                if free and n_hi[b]:
                    c.k_hi[b, h, self.free[b, h]], c.v_hi[b, h, self.free[b, h]] = nan, nan
        if parents is None:
            parents = [[-1 if i == 0 else int(torch.randint(max(-1, i - 5), i, (1,), generator=g, device="cuda"))
                        for i in range(nodes)] for _ in range(B)]
        self.parents = torch.tensor(parents, dtype=torch.int32, device="cuda").view(B, nodes)
        make = (lambda h: r(B, nodes, h, 128).to(torch.bfloat16).transpose(1, 2)) if major else \
            (lambda h: r(B, h, nodes, 128).to(torch.bfloat16))
        self.q, self.k, self.v = make(Hq), make(Hkv), make(Hkv)
        self.see = see_brute(parents)
        for b in range(B):
            for i in range(nodes):
                if not self.see[b][i]:
                    self.k[b, :, i], self.v[b, :, i] = nan, nan
        self.lens = pkg.Lengths(None if n_hi == [hi_cap] * B else self.dev(n_hi), self.dev(n_lo), self.free)

    def dev(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def masks(self):
        m = torch.full((self.shape.batch, self.N, 4), 77, dtype=torch.int32, device="cuda")
        pkg.mikv_tree_masks(m, self.parents)
        return m

    def used(self, b, h):
        """The slots that hold a token."""
        s = torch.arange(self.n_hi[b], device="cuda")
        return s[s != self.free[b, h]] if self.free is not None else s


def see_brute(parents):
    """[B][N] lists of what each node sees (empty: padding)."""
    out = []
    for row in parents:
        seen = []
        for i, p in enumerate(row):
            if p < -1 or p >= i or (p >= 0 and not seen[p]):
                seen.append([])
            else:
                seen.append((seen[p] if p >= 0 else []) + [i])
        out.append(seen)
    return out


def attention(d: Drafts, b, hq, scale=1 / math.sqrt(128), out_dtype=torch.bfloat16):
    """(out [N, 128], lse [N], bounds of both) of one query head.

    Bounds: scores of bf16 keys are exact products summed in fp32; a retained key is rounded at most twice to fp16 on its
    way (dequantized, divided by the balancer; subnormals: 2^-25 each), its query is exact; weights are then off by a
    factor e^(2 E), by 2^-19 for the exponential and the sums, and by their rounding to bf16 or fp16; retained values are
    rounded to fp16 once; fp16 weights lose what lies 2^-33 below the largest; the output is rounded once. (Of few rows
    the keys are not rounded, and a weight is rounded once more with its row's scale: 2^-11 of scale * code, which over the
    rows of these tests stays inside the same terms.)"""
    h, c = hq // d.G, d.cache
    q = d.q[b, hq].double()
    N, n_lo = d.N, d.n_lo[b]
    used = d.used(b, h)
    bits = d.shape.bits
    parts = [(c.k_hi[b, h, used].double(), c.v_hi[b, h, used].double())]
    kb = torch.zeros(0, 128, dtype=torch.float64, device="cuda")
    if bits and n_lo:
        bal = c.balancer[h].double() if c.balancer is not None else torch.ones(128, dtype=torch.float64, device="cuda")
        kb = values_of(c.k_codes[b, h, :n_lo], c.k_params[b, h, :n_lo], bits) / bal
        parts.append((kb, values_of(c.v_codes[b, h, :n_lo], c.v_params[b, h, :n_lo], bits)))
    real = torch.tensor([bool(x) for x in d.see[b]], device="cuda")
    see = torch.zeros(N, N, dtype=torch.bool)
    for i, x in enumerate(d.see[b]):
        see[i, x] = True
    see = see.cuda()
    kt, vt = (torch.where(real[:, None], x[b, h].double(), 0.0) for x in (d.k, d.v))
    parts.append((kt, vt))
    k, v = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
    n0, n1 = len(used), len(used) + len(kb)
    mask = torch.ones(N, len(k), dtype=torch.bool, device="cuda")
    mask[:, n1:] = see
    s = scale * (q @ k.T)
    E = scale * ACC_GAMMA * (q.abs() @ k.abs().T) + 2.0 ** -21 * s.abs()
    if n1 > n0:
        inv = 1 / bal
        E[:, n0:n1] += scale * (2.02 * U16 * (q.abs() @ kb.abs().T) + 2.0 ** -25 * (q.abs() @ (1 + inv))[:, None])
        # elements of a query below 2^-24 of its largest may be lost
        E[:, n0:n1] += scale * 2.0 ** -24 * q.abs().amax(1)[:, None] * kb.abs().sum(1)
    s = s.masked_fill(~mask, -math.inf)
    lse = torch.logsumexp(s, dim=1)
    w = torch.exp(s - lse[:, None])
    w = torch.where(real[:, None], w, 0.0)
    Em = torch.where(w > 2.0 ** -60, E, 0.0).amax(dim=1)
    out = w @ v
    rel = torch.full((len(k),), UNIT[torch.bfloat16], dtype=torch.float64, device="cuda")
    rel[n0:n1] = 2.02 * U16
    wide = (torch.expm1(2 * Em) + 2.0 ** -19)[:, None]
    inner = 2 * (w @ (v.abs() * rel[:, None]) + wide * (w @ v.abs())) + 2.0 ** -24
    if n1 > n0:
        inner = inner + n1 * 2.0 ** -33 * v[n0:n1].abs().amax(0)
    bound = inner + UNIT[out_dtype] * (out.abs() + inner)
    lse_bound = Em + 2.0 ** -19 + 2.0 ** -22 * lse.abs()
    lse = torch.where(real, lse, -math.inf)
    return out, lse, bound, torch.where(real, lse_bound, 0.0)


def near(got, want, bound, what):
    g = got.double()
    fin = torch.isfinite(want)
    assert bool((torch.isfinite(g) == fin).all()), f"{what}: finite where it should not be, or the reverse"
    assert bool((g[~fin] == want[~fin]).all()), what
    err, b = (g - want).abs()[fin], bound.expand_as(want)[fin]
    assert bool((err <= b).all()), f"{what}: {float((err / b.clamp(min=1e-300)).max()):.3f} of the bound"


def run(d: Drafts, out_dtype=torch.bfloat16, ws=None, lens=None, masks=None, major=True, **kw):
    B, Hq, N = d.shape.batch, d.shape.heads_q, d.N
    shape = (B, N, Hq, 128) if major else (B, Hq, N, 128)
    out = torch.full(shape, math.nan, dtype=out_dtype, device="cuda")
    out = out.transpose(1, 2) if major else out
    lse = torch.full((B, Hq, N), math.nan, device="cuda")
    ws = torch.zeros(pkg.mikv_tree_workspace_bytes(d.shape, N), dtype=torch.uint8, device="cuda") if ws is None else ws
    pkg.mikv_tree_attention(d.cache, d.masks() if masks is None else masks, d.q, d.k, d.v, out, ws,
                            lens=d.lens if lens is None else lens, lse=lse, **kw)
    pkg.mikv_workspace_check(ws)
    return out, lse


def check(d: Drafts, out, lse, heads=None, batch=None, **kw):
    for b in range(d.shape.batch) if batch is None else batch:
        for hq in range(d.shape.heads_q) if heads is None else heads:
            o, e, ob, eb = attention(d, b, hq, out_dtype=out.dtype, **kw)
            near(out[b, hq], o, ob, f"out b{b} h{hq}")
            near(lse[b, hq], e, eb, f"lse b{b} h{hq}")
