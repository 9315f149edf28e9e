"""Rotary positions on the GPU against the formula in 64 bits: types, pair layouts, part of the head, strides,
positions from negative to the largest, the transposed map as the gradient, scaled frequencies."""
import math

import pytest
import torch

import paper_2402_18096_gb300 as pkg
from paper_2402_18096_gb300.prompt import rotary_frequencies

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def turned(x, pos, freqs, layout, amplitude=1.0, inverse=False):
    """x [B, H, T, d], pos [B, T] in 64 bits; also the size |x| + |x'| of each pair (for the bounds)."""
    r = 2 * len(freqs)
    a = pos.double()[:, None, :, None] * torch.tensor(freqs, dtype=torch.float64, device=x.device)
    if inverse:
        a = -a
    c, s = amplitude * torch.cos(a), amplitude * torch.sin(a)
    xd = x.double()
    y, size = xd.clone(), xd.abs()
    one, two = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    p, q = xd[..., one], xd[..., two]
    y[..., one], y[..., two] = p * c - q * s, p * s + q * c
    size[..., one] = size[..., two] = abs(amplitude) * (p.abs() + q.abs())
    return y, size


def check(got, x, pos, freqs, layout, amplitude=1.0, inverse=False):
    """The angle is off by at most 2^-32 turns plus one rounding to fp32 (2^-24 of at most pi), cosine and sine by
    2^-22, the products and the sum round three times: 2^-20 of |x| + |x'| covers them; then one rounding."""
    y, size = turned(x, pos, freqs, layout, amplitude, inverse)
    # (the 64-bit reference forms pos * freq with 53 bits: 2^-53 of up to 2^31 radians, times the size)
    bound = (2.0 ** -20 + 2.0 ** -53 * pos.abs().max().item()) * size + UNIT[x.dtype] * y.abs()
    if x.dtype == torch.float16:
        bound = bound + 2.0 ** -25
    r = 2 * len(freqs)
    assert torch.equal(got[..., r:], x[..., r:])  # copied, bit for bit
    err = (got.double() - y).abs()
    assert bool((err <= bound).all()), float((err / bound.clamp(min=1e-30)).max())


def tensor(shape, dtype, token_major, gen):
    B, H, T, d = shape
    if token_major:
        return torch.randn(B, T, H, d, generator=gen, device="cuda").to(dtype).transpose(1, 2)
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [128, 64, 2, 10, 96])
@pytest.mark.parametrize("B,Hq,Hk,T", [(1, 1, 1, 1), (3, 5, 2, 7), (2, 8, 2, 130)])
def test_against_formula(dtype, layout, rot, B, Hq, Hk, T):
    g = gen(rot + T)
    q = tensor((B, Hq, T, 128), dtype, T % 2 == 0, g)
    k = tensor((B, Hk, T, 128), dtype, False, g)
    pos = torch.randint(0, 40000, (B, T), generator=g, device="cuda", dtype=torch.int32)
    f = rotary_frequencies(rot)
    table = pkg.RotaryTable(rot_dim=rot, layout=layout)
    q_out, k_out = torch.empty(B, Hq, T, 128, dtype=dtype, device="cuda"), torch.empty_like(k)
    pkg.mikv_rotary(table, q, k, q_out, k_out, positions=pos)
    check(q_out, q, pos, f, layout)
    check(k_out, k, pos, f, layout)
    # the transposed map, and in place with a running start
    pkg.mikv_rotary(table, q, None, q_out, positions=pos, inverse=True)
    check(q_out, q, pos, f, layout, inverse=True)
    x = k.clone()
    pkg.mikv_rotary(table, x, start=1234)
    check(x, k, (1234 + torch.arange(T, device="cuda")).expand(B, T), f, layout)


def test_unaligned_and_odd_strides():
    """Elements at any alignment: a slice one element into a wider tensor, rows of 131 elements."""
    g = gen(3)
    wide = torch.randn(2, 3, 9, 131, generator=g, device="cuda").to(torch.bfloat16)
    x = wide[..., 1:129]
    pos = torch.arange(9, device="cuda", dtype=torch.int32).expand(2, 9).contiguous()
    before = wide.clone()
    out = torch.empty(2, 3, 9, 128, dtype=torch.bfloat16, device="cuda")
    pkg.mikv_rotary(pkg.RotaryTable(), x, None, out, positions=pos)
    check(out, x, pos, rotary_frequencies(128), "half")
    pkg.mikv_rotary(pkg.RotaryTable(), x, positions=pos)
    assert torch.equal(x, out)
    assert torch.equal(wide[..., 0], before[..., 0]) and torch.equal(wide[..., 129:], before[..., 129:])


def test_extreme_positions():
    pos = torch.tensor([[0, 1, -1, -40000, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1]], dtype=torch.int32, device="cuda")
    x = torch.randn(1, 2, 7, 128, generator=gen(4), device="cuda")
    out = torch.empty_like(x)
    pkg.mikv_rotary(pkg.RotaryTable(), x, None, out, positions=pos)
    check(out, x, pos, rotary_frequencies(128), "half")


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                     dict(scaling="bands", factor=8.0, trained=2048)])
def test_scaled_for_long_contexts(scaling):
    f = rotary_frequencies(128, 10000.0, **scaling)
    plain = rotary_frequencies(128)
    if scaling["scaling"] == "linear":
        assert all(a == b / 4.0 for a, b in zip(f, plain))
    else:  # the fastest pair is kept, the slowest slowed by the factor
        assert f[0] == plain[0] and math.isclose(f[-1], plain[-1] / 8.0, rel_tol=1e-12)
        assert all(a <= b * (1 + 1e-12) for a, b in zip(f, plain))
    x = torch.randn(1, 4, 33, 128, generator=gen(5), device="cuda")
    pos = (100000 + torch.arange(33, device="cuda", dtype=torch.int32))[None]
    out = torch.empty_like(x)
    pkg.mikv_rotary(pkg.RotaryTable(amplitude=1.25, **scaling), x, None, out, positions=pos.contiguous())
    check(out, x, pos, f, "half", amplitude=1.25)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_gradient(layout):
    """The inverse map is the gradient: <R x, y> = <x, R' y>, and differences of <R x, y> in 64 bits agree."""
    g = gen(6)
    x, y = (torch.randn(2, 3, 5, 128, generator=g, device="cuda") for _ in range(2))
    table = pkg.RotaryTable(rot_dim=64, layout=layout, amplitude=0.75)
    grad, fwd = torch.empty_like(x), torch.empty_like(x)
    pkg.mikv_rotary(table, y, None, grad, start=77, inverse=True)
    pkg.mikv_rotary(table, x, None, fwd, start=77)
    a, b = float((fwd.double() * y.double()).sum()), float((x.double() * grad.double()).sum())
    assert abs(a - b) <= 2.0 ** -18 * float((x.abs() * y.abs()).sum() * 2)
    pos = (77 + torch.arange(5, device="cuda")).expand(2, 5)
    f = rotary_frequencies(64)
    step = torch.randn(2, 3, 5, 128, generator=g, device="cuda").double()

    def loss(z):
        return (turned(z, pos, f, layout, 0.75)[0] * y.double()).sum()

    diff = (loss(x.double() + step) - loss(x.double() - step)) / 2  # linear: the difference is exact
    assert abs(float(diff - (grad.double() * step).sum())) <= 2.0 ** -18 * float((step.abs() * y.abs()).sum() * 2)


def test_other_stream_and_repeat():
    x = torch.randn(2, 8, 300, 128, generator=gen(7), device="cuda").to(torch.bfloat16)
    table = pkg.RotaryTable()
    a, b = torch.empty_like(x), torch.empty_like(x)
    pkg.mikv_rotary(table, x, None, a, start=5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pkg.mikv_rotary(table, x, None, b, start=5)
    side.synchronize()
    assert torch.equal(a, b)


def test_wrong_arguments_raise():
    x = torch.zeros(1, 2, 3, 128, device="cuda")
    table = pkg.RotaryTable()
    with pytest.raises(ValueError):
        pkg.mikv_rotary(table, x, None, torch.zeros(1, 2, 3, 64, device="cuda"))
    with pytest.raises(ValueError):
        pkg.mikv_rotary(table, x, None, x.half())
    with pytest.raises(ValueError):
        pkg.mikv_rotary(table, x, positions=torch.zeros(1, 3, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        pkg.mikv_rotary(table, x.transpose(2, 3))
    with pytest.raises(ValueError):
        pkg.RotaryTable(layout="thirds")
    with pytest.raises(ValueError):
        pkg.RotaryTable(rot_dim=130)
    with pytest.raises(pkg.MikvError):
        pkg.mikv_rotary(table, torch.zeros(1, 2, 3, 64, device="cuda"))
