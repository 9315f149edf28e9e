"""The attention kernels where every CTA works through many items: more row tiles than six rounds of SMs in each layout
of rows, items without keys among them, heads that are taken in groups with a smaller last one; and values that are no
numbers in every layout."""
import math

import pytest
import torch

import paper_2402_18096_gb300 as pkg
from test_gpu_prompt import BF, FH, causal_spans, check_prefix, check_prompt, gen, make, prefix, prompt, slopes_of

pytestmark = pytest.mark.gpu


def sampled(q, k, v, out, lse, spans, pairs, **kw):
    """check_prompt of the (batch row, query head) pairs; everything else at least written."""
    assert not bool(torch.isnan(out).any()) and not bool(torch.isnan(lse).any())
    for b, h in pairs:
        one = slice(b, b + 1)
        check_prompt(q[one], k[one], v[one], out[one], lse[one], spans[one], heads=[h], **kw)


# (B, Hq, Hkv, tq, tk): row pairs, single row tiles, rows that stand in the tile four times
MANY = [(20, 32, 16, 300, 300), (60, 32, 16, 50, 500), (64, 16, 16, 9, 700)]


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s)))
def test_many_row_tiles(shape, dtype):
    B, Hq, Hkv, tq, tk = shape
    g = gen(tq)
    q, k, v = (make(g, (B, H, T, 128), dtype, big=big) for H, T, big in ((Hq, tq, False), (Hkv, tk, True), (Hkv, tk, False)))
    rows = {300: 3, 50: 1, 9: 1}[tq]
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert B * Hkv * rows > 6 * sms
    pairs = [(0, 0), (1, 7), (B // 2, 3), (B - 2, Hq - 1), (B - 1, 0), (B - 1, Hq - 1)]
    out, lse = prompt(q, k, v)
    sampled(q, k, v, out, lse, causal_spans(B, tq, tk, tk - tq), pairs, q_start=tk - tq)
    again, lse2 = prompt(q, k, v)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("cap,bias", [(0.0, True), (20.0, False)])
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s)))
def test_many_row_tiles_some_without_keys(shape, cap, bias):
    """Spans that leave whole batch rows, and runs of queries in others, without keys: items without tiles in between."""
    B, Hq, Hkv, tq, tk = shape
    g = gen(tk)
    q, k, v = make(g, (B, Hq, tq, 128), BF), make(g, (B, Hkv, tk, 128), BF), make(g, (B, Hkv, tk, 128), BF)
    a = torch.randint(0, tk + 1, (B, tq, 2), generator=g, device="cuda", dtype=torch.int32).sort(dim=2).values.contiguous()
    a[1::3] = 0
    a[2:4] = 0
    a[::2, :tq // 2] = 0
    a[-1] = torch.tensor([0, tk], device="cuda")
    sl = slopes_of(Hq) if bias else None
    kw = dict(softcap=cap, slopes=sl, causal=False, q_start=0)
    out, lse = prompt(q, k, v, spans=a, **kw)
    pairs = [(0, 0), (1, 5), (2, 1), (B // 2, 3), (B - 2, Hq - 1), (B - 1, Hq - 1)]
    sampled(q, k, v, out, lse, a, pairs, cap=cap, slopes=sl)
    again, lse2 = prompt(q, k, v, spans=a, **kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("B,H,T", [(2, 40, 4096), (1, 37, 3999)])
def test_heads_in_groups(B, H, T, dtype):
    """More heads than have their keys in half of L2 together (32 at these lengths): full groups and a smaller last."""
    g = gen(H)
    q, k, v = make(g, (B, H, T, 128), dtype), make(g, (B, H, T, 128), dtype, big=True), make(g, (B, H, T, 128), dtype)
    out, lse = prompt(q, k, v)
    pairs = [(0, 0), (0, 31), (0, 32), (B - 1, H - 9), (B - 1, H - 1)]
    sampled(q, k, v, out, lse, causal_spans(B, T, T, 0), pairs)
    again, lse2 = prompt(q, k, v)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF, FH])
def test_many_prefixes(dtype):
    """Single tokens over more prefixes than six rounds of SMs, ragged lengths, none at all among them."""
    n, Hq, Hkv, P = 70, 32, 16, 300
    g = gen(n)
    q = torch.randn(2 * n, Hq, 128, generator=g, device="cuda").to(dtype)
    k, v = make(g, (n, Hkv, P, 128), dtype), make(g, (n, Hkv, P, 128), dtype)
    lens = torch.randint(0, P + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    lens[::5] = 0
    out, ml = prefix(q, k, v, lens=lens)
    assert not bool(torch.isnan(out).any()) and not bool(torch.isnan(ml).any())
    check_prefix(q, k, v, out, ml, lens)
    again, ml2 = prefix(q, k, v, lens=lens)
    assert torch.equal(out, again) and torch.equal(ml, ml2)


# one item or more in each layout: row pairs, one row tile, few rows; whole row tiles and shared keys
LAYOUTS = [(1, 8, 2, 200, 256), (1, 4, 1, 30, 256), (1, 2, 1, 4, 256), (1, 8, 2, 200, 4096), (1, 4, 1, 30, 4096),
           (1, 2, 1, 4, 4096)]


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("shape", LAYOUTS, ids=lambda s: "x".join(map(str, s)))
def test_visible_values_that_are_no_numbers(shape, bad):
    """Rows that see an infinity or NaN give one in its channel; in tiles that no mask cuts every other channel keeps its
    value, and rows that do not see it keep all of theirs."""
    B, Hq, Hkv, tq, tk = shape
    g = gen(tk + tq)
    q, k, v = make(g, (B, Hq, tq, 128), BF), make(g, (B, Hkv, tk, 128), BF), make(g, (B, Hkv, tk, 128), BF)
    at = 150
    v[:, 0, at, 3] = bad
    zero = v.clone()
    zero[:, 0, at, 3] = 0
    out, lse = prompt(q, k, v, causal=False)  # (whole tiles: no mask)
    clean, clean_lse = prompt(q, k, zero, causal=False)
    G = Hq // Hkv
    assert not bool(torch.isfinite(out[:, :G, :, 3]).any())
    rest = [c for c in range(128) if c != 3]
    assert torch.equal(out[:, :, :, rest], clean[:, :, :, rest])
    assert torch.equal(out[:, G:], clean[:, G:]) and torch.equal(lse, clean_lse)
    # every other row stops short of the key, inside its tile
    a = torch.tensor([0, tk], dtype=torch.int32, device="cuda").expand(B, tq, 2).contiguous()
    a[:, ::2, 1] = at
    out, lse = prompt(q, k, v, spans=a)
    clean, clean_lse = prompt(q, k, zero, spans=a)
    assert not bool(torch.isfinite(out[:, :G, 1::2, 3]).any())
    assert torch.equal(out[:, :, ::2], clean[:, :, ::2]) and torch.equal(lse, clean_lse)
    assert torch.equal(out[:, G:], clean[:, G:])
