"""Tree attention over retained values of any size: value scales far below 1, of 0, and rising along a request, in small
caches and in large ones (few rows have a kernel of their own there), against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2402_18096_gb300 as pkg
from _tree_ref import ACC_GAMMA, U16, UNIT, Drafts, codes_of, near, run, values_of

pytestmark = pytest.mark.gpu

F32 = torch.float32


@pytest.fixture(params=[0, (1 << 18) + 1], ids=["small", "roomy"])
def few(request, monkeypatch):
    """Whether few rows go to their own kernel."""
    monkeypatch.setattr(Drafts, "tokens", request.param)
    return request.param > 0


def reference(d, b, hq, tile):
    """(out, lse, bounds) of one query head; `tile`: values are rounded to fp16 tiles.

    Bounds of out. A retained value is alpha * code + beta; with A = |alpha| code and B = |beta| the weights P are rounded to
    fp16 (2^-11 of A + B) and either P alpha once more (2^-11 of A) or the value (2^-11 of it, at least 2^-25): 2.02 U16
    (A + B) holds both, and their product. Weights of slots and nodes are rounded to bf16. Weights below 2^-14 are rounded
    to multiples of 2^-24 while the sum is 2^8 at least: 2^-33 a key. So are P alpha in units of the power of two at or
    below the largest scale (2^-14 at least), and P in units of that power where it is above 1. `wide`: the scores' errors
    E as factors of the weights, in the numerator and the sum. Products are summed in fp32, 16 keys at a time."""
    h, c, N, n_lo, scale = hq // d.G, d.cache, d.N, d.n_lo[b], 1 / math.sqrt(128)
    q, used = d.q[b, hq].double(), d.used(b, h)
    bal = c.balancer[h].double()
    kb = values_of(c.k_codes[b, h, :n_lo], c.k_params[b, h, :n_lo], d.shape.bits) / bal
    p = c.v_params[b, h, :n_lo].double().repeat_interleave(d.shape.group, -2)
    A = p[..., 0].abs() * codes_of(c.v_codes[b, h, :n_lo], d.shape.bits)
    k = torch.cat([c.k_hi[b, h, used].double(), kb, d.k[b, h].double()])
    v_hi, v_t = c.v_hi[b, h, used].double(), d.v[b, h].double()
    v = torch.cat([v_hi, values_of(c.v_codes[b, h, :n_lo], c.v_params[b, h, :n_lo], d.shape.bits), v_t])
    size = torch.cat([v_hi.abs(), A + p[..., 1].abs(), v_t.abs()])
    n0, n1 = len(used), len(used) + n_lo
    mask = torch.ones(N, len(k), dtype=torch.bool, device="cuda")
    mask[:, n1:] = False
    for i, seen in enumerate(d.see[b]):
        mask[i, [n1 + j for j in seen]] = True
    s = scale * (q @ k.T)
    E = scale * ACC_GAMMA * (q.abs() @ k.abs().T) + 2.0 ** -21 * s.abs()
    E[:, n0:n1] += scale * (2.02 * U16 * (q.abs() @ kb.abs().T) + 2.0 ** -25 * (q.abs() @ (1 + 1 / bal))[:, None])
    E[:, n0:n1] += scale * 2.0 ** -24 * q.abs().amax(1)[:, None] * kb.abs().sum(1)
    s = s.masked_fill(~mask, -math.inf)
    lse = torch.logsumexp(s, dim=1)
    w = torch.exp(s - lse[:, None])
    Em = torch.where(w > 2.0 ** -60, E, 0.0).amax(dim=1)
    out = w @ v
    rel = torch.full((len(k), 1), UNIT[torch.bfloat16], dtype=torch.float64, device="cuda")
    rel[n0:n1] = 2.02 * U16
    rel += 2.0 ** -23 * (len(k) / 16 + 16)
    bound = w @ (size * rel) + 2 * (torch.expm1(2 * Em) + 2.0 ** -19)[:, None] * (w @ size)
    if n_lo:
        top = max(float(p[..., 0].abs().max()), 2.0 ** -14)
        bound = bound + n_lo * 2.0 ** -33 * (max(top, 1.0) * size[n0:n1].amax(0) + top * (2 ** d.shape.bits - 1))
    if tile:
        bound = bound + 2.0 ** -25
    bound = bound + UNIT[F32] * (out.abs() + bound)
    return out, lse, bound, Em + 2.0 ** -19 + 2.0 ** -22 * lse.abs()


def check(d, few):
    out, lse = run(d, F32)
    for b in range(d.shape.batch):
        for hq in range(d.shape.heads_q):
            o, e, ob, eb = reference(d, b, hq, tile=not few or d.N * d.G > 16)
            near(out[b, hq], o, ob, f"out b{b} h{hq}")
            near(lse[b, hq], e, eb, f"lse b{b} h{hq}")


def of_size(d, factor):
    """The same requests with all their values times `factor` (a power of two; per retained row where it is a tensor)."""
    rows = factor if torch.is_tensor(factor) else torch.full((d.shape.lo_cap,), factor, device="cuda")
    d.cache.v_params.copy_((d.cache.v_params.float() * rows[:, None, None]).half())
    least = float(rows.min())
    d.cache.v_hi.mul_(least)
    d.v.mul_(least)


HEADS = [(2, 2, 5), (4, 2, 6), (4, 1, 30)]  # (query heads, KV heads, nodes): 5 rows, 12, 120
CODES = [(2, 32), (2, 64), (2, 128), (3, 32), (3, 64), (3, 128), (4, 32), (4, 64), (4, 128)]


@pytest.mark.parametrize("power", [-5, -7, -8, -10, -14])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("bits,group", CODES)
def test_values_of_any_size(few, bits, group, heads, power):
    Hq, Hkv, N = heads
    d = Drafts(bits + group - power, 2, Hq, Hkv, N, 40, 608, bits, group, n_lo=[608, 37])
    of_size(d, 2.0 ** power)
    check(d, few)


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("bits,group", [(2, 32), (3, 128), (4, 64)])
@pytest.mark.parametrize("which", ["scales", "first scales", "all"])
def test_values_without_a_scale(few, bits, group, heads, which):
    """Scales of 0 in every row, in the first rows of a request, and values of 0."""
    Hq, Hkv, N = heads
    d = Drafts(3 * bits + group, 2, Hq, Hkv, N, 40, 1504, bits, group, n_lo=[1504, 90])
    for b, n in enumerate(d.n_lo):
        rows = d.cache.v_params[b, :, :80 if which == "first scales" else n]
        rows[..., 0] = 0
        if which == "all":
            rows[..., 1] = 0
    check(d, few)


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("bits,group", [(2, 32), (3, 64), (4, 128)])
@pytest.mark.parametrize("falling", [False, True], ids=["rising", "falling"])
def test_values_whose_size_changes_along_a_request(few, bits, group, heads, falling):
    """Rows from 2^-13 to 2^-1 of the usual size, by 2^2 every 96 rows, and the reverse."""
    Hq, Hkv, N = heads
    d = Drafts(5 * bits + group, 2, Hq, Hkv, N, 40, 608, bits, group, n_lo=[608, 300])
    step = torch.div(torch.arange(d.shape.lo_cap, device="cuda"), 96, rounding_mode="floor").clamp(max=6)
    of_size(d, torch.exp2(2.0 * (6 - step if falling else step) - 13))
    check(d, few)
