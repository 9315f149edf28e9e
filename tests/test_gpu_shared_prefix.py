"""The shared-prefix layer: decode steps over a bf16 prefix and a mixed-precision cache of own tokens, against attention
over everything in 64 bits; with no prefix it does what the fused decode step does; the example runs."""
import os
import sys

import pytest
import torch

import paper_2402_18096_gb300 as pkg
from paper_2402_18096_gb300.layer import MixedPrecisionLayer, SharedPrefixLayer
import _attn_ref as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def make(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def turned(table, x, start):
    y = x.clone()
    pkg.mikv_rotary(table, y, start=start)
    return y


def test_prompts_and_steps_against_full_attention():
    """An all-important own cache (ratio 1: nothing is quantized at the prompt, one token per step): the prompt outputs
    and the first step equal attention over prefix and own tokens."""
    B, Hq, Hkv, P, T = 3, 8, 2, 300, 70
    g = torch.Generator(device="cuda").manual_seed(3)
    table = pkg.RotaryTable()
    q0, k0, v0 = (make(g, 1, h, P, 128) for h in (Hq, Hkv, Hkv))
    q, k, v = (make(g, B, h, T, 128) for h in (Hq, Hkv, Hkv))
    kq, kk = turned(table, q, P), turned(table, k, P)
    pk = turned(table, k0, 0)
    shape = pkg.shape_for_context(B, Hq, Hkv, 2, 32, T, 1.0, 4)
    out0 = torch.empty(1, Hq, P, 128, dtype=torch.bfloat16, device="cuda")
    out1 = torch.empty(B, Hq, T, 128, dtype=torch.bfloat16, device="cuda")
    layer = SharedPrefixLayer.from_prompts(shape, table, (q0, k0, v0), (q, k, v), out0, out1)
    scale = 128 ** -0.5
    for b in range(B):
        for h in range(Hq):
            keys, vals = torch.cat([pk[0, h // 4], kk[b, h // 4]]), torch.cat([v0[0, h // 4], v[b, h // 4]])
            mask = torch.arange(P + T, device="cuda") <= P + torch.arange(T, device="cuda")[:, None]
            o, _, bound, _ = ref.attention(kq[b, h], keys, vals, mask, scale)
            assert bool(((out1[b, h].double() - o).abs() <= bound).all())
    qn, kn, vn = (make(g, B, h, 128) for h in (Hq, Hkv, Hkv))
    tq, tk = turned(table, qn[:, :, None], P + T)[:, :, 0], turned(table, kn[:, :, None], P + T)[:, :, 0]
    out = torch.empty(B, Hq, 128, dtype=torch.bfloat16, device="cuda")
    layer.step(qn, kn, vn, out)
    assert torch.equal(qn, tq)
    for b in range(B):
        for h in range(Hkv):
            keys = torch.cat([pk[0, h], kk[b, h], tk[b, h][None]])
            vals = torch.cat([v0[0, h], v[b, h], vn[b, h][None]])
            rows = tq[b, 4 * h:4 * h + 4]
            o, e, bound, eb = ref.attention(rows, keys, vals, torch.ones(4, len(keys), dtype=torch.bool, device="cuda"),
                                            scale)
            vmax = float(vals.double().abs().max())  # (the own part's documented bound is 2e-3 of it)
            assert bool(((out[b, 4 * h:4 * h + 4].double() - o).abs() <= bound + 2e-3 * vmax).all())
            assert bool(((layer.ml[b, 4 * h:4 * h + 4, 0].double() - e).abs() <= eb + 2.0 ** -16).all())
    assert layer.own.n_lo == 1 and layer.own.pos == T + 1


def test_without_a_prefix_it_is_the_fused_step():
    B, Hq, Hkv, T, steps = 2, 8, 2, 200, 5
    g = torch.Generator(device="cuda").manual_seed(4)
    table = pkg.RotaryTable()
    k, v, qp = make(g, B, Hkv, T, 128), make(g, B, Hkv, T, 128), make(g, B, Hq, T, 128)
    shape = pkg.shape_for_context(B, Hq, Hkv, 3, 64, T, 0.2, steps)
    one, two = (MixedPrecisionLayer.from_prefill(shape, k, v, None, qp) for _ in range(2))
    none = torch.empty(1, Hkv, 0, 128, dtype=torch.bfloat16, device="cuda")
    shared = SharedPrefixLayer(one, none, none, table)
    a, b = torch.empty(B, Hq, 128, device="cuda"), torch.empty(B, Hq, 128, device="cuda")
    for i in range(steps):
        q, kn, vn = make(g, B, Hq, 128), make(g, B, Hkv, 128), make(g, B, Hkv, 128)
        tq, tk = turned(table, q[:, :, None], T + i)[:, :, 0], turned(table, kn[:, :, None], T + i)[:, :, 0]
        shared.step(q, kn, vn, a)
        two.step(tq.contiguous(), tk.contiguous(), vn, b)
        assert torch.equal(a, b)
        assert torch.equal(one.slots, two.slots)
    n = one.n_lo
    assert n == two.n_lo
    assert torch.equal(one.cache.k_codes[:, :, :n], two.cache.k_codes[:, :, :n])
    assert torch.equal(one.cache.lo_tok[:, :, :n], two.cache.lo_tok[:, :, :n])


def test_coded_important_set_is_refused():
    shape = pkg.shape_for_context(1, 4, 2, 2, 64, 64, 0.25, 1, hi_bits=8)
    own = MixedPrecisionLayer(shape)
    k = torch.zeros(1, 2, 16, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        SharedPrefixLayer(own, k, k, pkg.RotaryTable())


def test_example_runs():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import shared_prompt
    finally:
        sys.path.pop(0)
    outs, us = shared_prompt.run(requests=3, prefix=257, own=65, steps=4, heads_q=8, heads_kv=2)
    assert bool(torch.isfinite(outs).all()) and us > 0
