"""Trees of drafted tokens on the GPU: their masks, and their attention over mixed-precision caches against the definition
in 64 bits (bounds of _tree_ref.attention), at the sizes, lengths and masks where it can go wrong."""
import math
import random

import pytest
import torch

import paper_2402_18096_gb300 as pkg
from _tree_ref import Drafts, check, gen, run, see_brute

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True, params=[0, (1 << 18) + 1], ids=["small", "roomy"])
def room(request, monkeypatch):
    """Caches as small as what they hold, and large ones: few rows have a kernel of their own there."""
    monkeypatch.setattr(Drafts, "tokens", request.param)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 100, 128])
def test_masks_and_positions(n):
    rng = random.Random(n)
    rows = [[i - 1 for i in range(n)], [-1] * n, [(i - 1) // 2 if i else -1 for i in range(n)],
            [rng.randrange(-2, max(i, 1) + 1) for i in range(n)], [-2] * n, [rng.choice((-5, 127, n, -1)) for _ in range(n)]]
    parents = torch.tensor(rows, dtype=torch.int32, device="cuda")
    masks = torch.full((len(rows), n, 4), 9, dtype=torch.int32, device="cuda")
    pos = torch.empty(len(rows), n, dtype=torch.int32, device="cuda")
    first = torch.arange(len(rows), dtype=torch.int32, device="cuda") * 1000
    pkg.mikv_tree_masks(masks, parents, positions=pos, first=first)
    for b, row in enumerate(see_brute(rows)):
        for i, seen in enumerate(row):
            want = sum(1 << j for j in seen)
            got = sum((int(w) & 0xffffffff) << (32 * j) for j, w in enumerate(masks[b, i].tolist()))
            assert got == want, (b, i)
            assert int(pos[b, i]) == 1000 * b + max(len(seen) - 1, 0)
    pkg.mikv_tree_masks(masks, parents, positions=pos, start=7)
    assert int(pos[1].min()) == int(pos[1].max()) == 7


# (B, Hq, Hkv, nodes, hi_cap, lo_cap, bits, group): one token; nothing but the tree; tiles of keys and rows exactly, one
# past, one short; rows of several tiles; every code width and group
SHAPES = [(1, 1, 1, 1, 1, 0, 2, 32), (2, 4, 4, 1, 2, 16, 2, 64), (1, 2, 1, 3, 0, 128, 3, 32), (1, 8, 1, 16, 128, 144, 4, 128),
          (2, 4, 2, 5, 129, 256, 2, 32), (1, 8, 1, 17, 300, 400, 3, 128), (1, 4, 4, 128, 127, 128, 4, 32),
          (1, 8, 1, 127, 260, 272, 3, 64), (3, 8, 2, 33, 513, 1040, 2, 128), (1, 8, 1, 128, 40, 640, 4, 64),
          (1, 8, 4, 64, 1000, 0, 2, 32), (2, 16, 2, 7, 50, 2064, 2, 32), (1, 4, 1, 65, 700, 3008, 4, 64),
          (1, 2, 2, 4, 384, 0, 0, 32), (5, 2, 1, 40, 100, 512, 0, 32)]


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_tree(shape, out_dtype):
    B, Hq, Hkv, N, hi, lo, bits, group = shape
    d = Drafts(sum(shape), B, Hq, Hkv, N, max(hi, 1), max(lo, 16), bits, group, n_hi=[hi] * B,
               n_lo=[lo if bits else 0] * B, free=hi > 0, balanced=N != 5)
    out, lse = run(d, out_dtype)
    check(d, out, lse)


@pytest.mark.parametrize("bits,group", [(2, 32), (2, 64), (3, 32), (3, 64), (3, 128), (4, 32), (4, 128), (0, 32)])
@pytest.mark.parametrize("G,N", [(1, 9), (4, 40)])
def test_ragged_requests(bits, group, G, N):
    """Requests of any lengths, down to none at all; padding nodes; requests whose nodes are all padding."""
    rng = random.Random(100 * bits + G)
    hi, lo = 400, 1504
    n_hi = [hi, 1, 0, 128, 129, 257, 33, 0, 399]
    n_lo = [lo, 0, 1, 128, 127, 900, 0, 0, 1281] if bits else [0] * 9
    parents = []
    for b in range(9):
        used = N if b in (0, 7) else 0 if b == 3 else rng.randrange(1, N + 1)
        parents.append([rng.randrange(-1, i) if i < used else -2 for i in range(N)])
    d = Drafts(bits + G, 9, 2 * G, 2, N, hi, lo, bits, group, n_hi=n_hi, n_lo=n_lo, parents=parents)
    out, lse = run(d)
    check(d, out, lse)
    empty = torch.tensor([[not x for x in row] for row in d.see], device="cuda")
    assert bool((out.transpose(1, 2)[empty] == 0).all()) and bool((lse.transpose(1, 2)[empty] == -math.inf).all())


def test_many_requests_and_items():
    """More row tiles than SMs, of lengths that change from one to the next."""
    rng = random.Random(3)
    B = 70
    n_hi, n_lo = [rng.randrange(0, 201) for _ in range(B)], [rng.choice((0, 5, 130, 500)) for _ in range(B)]
    d = Drafts(8, B, 16, 4, 11, 200, 512, 3, 64, n_hi=n_hi, n_lo=n_lo)
    out, lse = run(d)
    check(d, out, lse, heads=(0, 5, 15), batch=range(0, B, 3))


@pytest.mark.parametrize("N,G", [(3, 2), (100, 2), (128, 8)])
def test_long_context(N, G):
    """One request whose keys are shared out among all SMs."""
    d = Drafts(N, 1, G, 1, N, 2900, 30000 // 16 * 16, 2, 32, n_hi=[2801], n_lo=[29001])
    out, lse = run(d)
    check(d, out, lse)


@pytest.mark.parametrize("scale,outliers", [(1e-3, 1.0), (0.3, 8.0), (2.0, 8.0)])
def test_scales_and_large_scores(scale, outliers):
    """Nearly uniform weights, and scores of hundreds whose largest comes anywhere."""
    d = Drafts(5, 2, 4, 2, 20, 300, 704, 4, 32, outliers=outliers)
    out, lse = run(d, sm_scale=scale)
    check(d, out, lse, scale=scale)


@pytest.mark.parametrize("power", [-40, 40])
def test_large_and_small_queries(power):
    """Queries far outside fp16, with a scale that brings the scores back."""
    d = Drafts(6, 1, 2, 1, 6, 100, 304, 2, 64)
    d.q.mul_(2.0 ** power)
    scale = 2.0 ** -power / math.sqrt(128)
    out, lse = run(d, sm_scale=scale)
    check(d, out, lse, scale=scale)


def test_balancers_of_any_size():
    """Channels whose balancer is far from 1 (the keys they belong to as far)."""
    d = Drafts(7, 1, 4, 2, 6, 64, 208, 4, 32)
    bal = d.cache.balancer
    for i, e in enumerate((-18, -9, 9, 18)):  # by groups, so that the parameters follow
        bal[:, 32 * i:32 * i + 32] *= 2.0 ** e
        d.cache.k_params[..., i, :] = (d.cache.k_params[..., i, :].float() * 2.0 ** min(e, 9)).half()
    out, lse = run(d)
    check(d, out, lse)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_bad_value_touches_those_that_see_it(bad):
    parents = [[-1, 0, 0, 1, 1, 2, 2, 3, -1]]
    d = Drafts(9, 1, 4, 2, 9, 60, 208, 2, 32, parents=parents)
    clean, clean_lse = run(d)
    d.v[:, :, 2, 17] = bad
    out, lse = run(d)
    sees = torch.tensor([2 in x for x in d.see[0]], device="cuda")
    assert bool(torch.isnan(out[:, :, sees]).all()) and torch.equal(lse, clean_lse)
    assert torch.equal(out[:, :, ~sees], clean[:, :, ~sees])
    d.v[:, :, 2, 17] = 0
    d.k[:, :, 2, 3] = math.nan  # a key: its own scores alone
    out, lse = run(d)
    assert bool(torch.isnan(out[:, :, sees]).all()) and bool(torch.isnan(lse[:, :, sees]).all())
    assert bool(torch.isfinite(out[:, :, ~sees]).all())
    d.k[:, :, 2, 3] = 0
    d.q[:, 1, 4, 100] = bad  # a query: its own row alone
    out, _ = run(d)
    assert bool(torch.isnan(out[0, 1, 4]).all())
    rows = torch.ones(4, 9, dtype=torch.bool, device="cuda")
    rows[1, 4] = False
    assert bool(torch.isfinite(out[0][rows]).all())


def test_views():
    """Operands as views of one projection, the output into a wider buffer, head-major rows."""
    d = Drafts(10, 2, 8, 2, 12, 90, 208, 3, 32)
    p = torch.randn(2, 12, 8 + 4, 128, generator=gen(1), device="cuda").to(BF)
    d.q, d.k, d.v = (p[:, :, a:b].transpose(1, 2) for a, b in ((0, 8), (8, 10), (10, 12)))
    wide = torch.full((2, 12, 11, 128), 7.0, dtype=BF, device="cuda")
    out = wide[:, :, 1:9].transpose(1, 2)
    lse = torch.empty(2, 8, 12, device="cuda")
    ws = torch.zeros(pkg.mikv_tree_workspace_bytes(d.shape, 12), dtype=torch.uint8, device="cuda")
    pkg.mikv_tree_attention(d.cache, d.masks(), d.q, d.k, d.v, out, ws, lens=d.lens, lse=lse)
    check(d, out, lse)
    assert bool((wide[:, :, 0] == 7).all()) and bool((wide[:, :, 9:] == 7).all())
    out2, lse2 = run(d, major=False)
    assert torch.equal(out2, out.contiguous()) and torch.equal(lse2, lse)
    pkg.mikv_tree_attention(d.cache, d.masks(), d.q, d.k, d.v, out2, ws, lens=d.lens)  # no lse asked for
    assert torch.equal(out2, out.contiguous())


def test_without_lengths():
    """Every slot in use and no retained rows; one number of rows for all."""
    d = Drafts(11, 2, 4, 2, 6, 70, 304, 2, 32, free=False, n_lo=[0, 0])
    out, lse = run(d, lens=pkg.Lengths())
    check(d, out, lse)
    ws = torch.zeros(pkg.mikv_tree_workspace_bytes(d.shape, 6), dtype=torch.uint8, device="cuda")
    out2 = torch.empty_like(out)
    pkg.mikv_tree_attention(d.cache, d.masks(), d.q, d.k, d.v, out2, ws)
    assert torch.equal(out2, out)
    d = Drafts(11, 2, 4, 2, 6, 70, 304, 2, 32, free=False, n_lo=[200, 200])
    out, lse = run(d, lens=pkg.Lengths(n_lo=200))
    check(d, out, lse)


def test_lengths_beyond_the_cache(room, monkeypatch):
    """Lengths are held to the cache's capacity, free slots outside those in use are none."""
    lo = max(304, Drafts.tokens // 64 * 16 + 16)
    monkeypatch.setattr(Drafts, "tokens", 0)
    d = Drafts(12, 2, 4, 2, 6, 70, lo, 2, 32, free=False)
    d.lens = pkg.Lengths(d.dev([5000, 70]), d.dev([2 ** 31 - 1, lo]), torch.full((2, 2), 70, dtype=torch.int32, device="cuda"))
    out, lse = run(d)
    check(d, out, lse)
    d.n_hi, d.n_lo = [0, 70], [0, lo]
    d.lens = pkg.Lengths(d.dev([-3, 70]), d.dev([-1, lo]), torch.full((2, 2), -1, dtype=torch.int32, device="cuda"))
    out, lse = run(d)
    check(d, out, lse)


def test_same_bits_every_time_and_in_graphs():
    """Repeated calls, a shared workspace, two captured graphs of one workspace replayed in turn, another stream."""
    a = Drafts(13, 3, 8, 2, 21, 150, 1200, 2, 32, n_hi=[150, 20, 77], n_lo=[1200, 3, 700])
    b = Drafts(14, 1, 8, 2, 3, 150, 3008, 4, 64)
    ws = torch.zeros(max(pkg.mikv_tree_workspace_bytes(x.shape, x.N) for x in (a, b)), dtype=torch.uint8, device="cuda")
    want = [run(x) for x in (a, b)]
    outs = [(torch.zeros_like(o), torch.zeros_like(e)) for o, e in want]
    graphs = []
    side = torch.cuda.Stream()
    for x, (o, e) in zip((a, b), outs):
        m = x.masks()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            pkg.mikv_tree_masks(m, x.parents)
            pkg.mikv_tree_attention(x.cache, m, x.q, x.k, x.v, o, ws, lens=x.lens, lse=e)
        graphs.append((g, m))
    for _ in range(3):
        for (g, _), (o, e), w in zip(graphs, outs, want):
            o.fill_(3), e.fill_(3)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, w[0]) and torch.equal(e, w[1])
    with torch.cuda.stream(side):
        got = run(a, ws=ws)
    side.synchronize()
    assert torch.equal(got[0], want[0][0]) and torch.equal(got[1], want[0][1])


def test_offsets_past_32_bits():
    """A cache whose arrays pass 4 GB; the last request's rows lie behind that."""
    B, H, lo = 4, 34, 1 << 20
    s = pkg.Shape(B, H, H, 2, 32, 1, lo)
    d = Drafts(15, 1, 1, 1, 4, 1, 208, 2, 32)
    c = pkg.LayerCache(s)
    for name in ("k_codes", "v_codes", "k_params", "v_params"):
        getattr(c, name)[-1, -1, :208] = getattr(d.cache, name)[0, 0, :208]
    c.balancer = torch.ones(H, 128, device="cuda")
    c.balancer[-1] = d.cache.balancer[0]
    q, k, v = (torch.zeros(B, H, 4, 128, dtype=BF, device="cuda") for _ in range(3))
    q[-1, -1], k[-1, -1], v[-1, -1] = d.q[0, 0], d.k[0, 0], d.v[0, 0]
    masks = d.masks().expand(B, 4, 4).contiguous()
    lens = pkg.Lengths(torch.ones(B, dtype=torch.int32, device="cuda"), d.dev([0, 0, 0, 208]),
                       torch.zeros(B, H, dtype=torch.int32, device="cuda"))
    out, lse = torch.empty_like(q), torch.empty(B, H, 4, device="cuda")
    ws = torch.zeros(pkg.mikv_tree_workspace_bytes(s, 4), dtype=torch.uint8, device="cuda")
    pkg.mikv_tree_attention(c, masks, q, k, v, out, ws, lens=lens, lse=lse)
    pkg.mikv_workspace_check(ws)
    check(d, out[-1:, -1:], lse[-1:, -1:])


@pytest.mark.parametrize("bits,group", [(2, 32), (3, 64), (4, 128)])
def test_scales_of_either_sign_and_size(bits, group):
    """Parameters that no quantizer gives but the formula takes: negative scales, rows 2^12 apart."""
    d = Drafts(16 + bits, 2, 4, 2, 3, 40, 608, bits, group)
    g = gen(5)
    for x in (d.cache.k_params, d.cache.v_params):
        sign = torch.where(torch.rand(x.shape[:-1], generator=g, device="cuda") < 0.5, -1.0, 1.0)
        x[..., 0] = (x[..., 0].float() * sign).half()
    step = 2.0 ** (4 * torch.randint(-2, 2, d.cache.v_params.shape[:3], generator=g, device="cuda").float())
    d.cache.v_params.copy_((d.cache.v_params.float() * step[..., None, None]).half())
    for dt in (BF, F32):
        out, lse = run(d, dt)
        check(d, out, lse)
