"""What follows the attention of drafted tokens, on the GPU: importance of accepted paths (against 64 bits), their entry
into the cache (against the oracle's quantizer and a plain sort), copies of requests, and a run of all of it."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2402_18096_gb300 as pkg
from _tree_ref import Drafts, attention, check, gen, near, values_of
from paper_2402_18096_gb300.layer import DraftedLayer

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
ARRAYS = ("k_hi", "v_hi", "hi_tok", "acc", "k_codes", "v_codes", "k_params", "v_params", "lo_tok")


def path_tensor(rows, steps):
    return torch.tensor([(list(r) + [-1] * steps)[:steps] for r in rows], dtype=torch.int32, device="cuda")


def drafts(seed=1, B=4, Hq=8, Hkv=2, N=9, hi=150, lo=320, bits=2, group=32, **kw):
    parents = [[-1, 0, 1, 2, 3, 4, 5, 6, 7][:N]] * B
    return Drafts(seed, B, Hq, Hkv, N, hi, lo, bits, group, parents=parents, **kw)


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 1), (8, 2)])
@pytest.mark.parametrize("hi,steps", [(1, 1), (64, 3), (65, 9), (700, 2), (700, 9)])
def test_importance(Hq, Hkv, hi, steps):
    d = drafts(hi + steps, Hq=Hq, Hkv=Hkv, hi=hi, n_hi=[hi, 1, max(hi - 7, 0), 0])
    rows = [range(steps), [], [0, 1, 2, 99, 4][:steps], [3]]
    count = [steps, 0, min(steps, 3), 1]
    path = path_tensor(rows, steps)
    lse = 3 + torch.rand(4, Hq, d.N, generator=gen(2), device="cuda")
    lse[0, 0, 0] = -math.inf  # weighs nothing
    before = d.cache.acc.clone()
    gained = torch.full((4, Hkv, steps), math.nan, device="cuda")
    pkg.mikv_path_importance(d.cache, path, d.q, d.k, lse, gained, lens=d.lens)
    scale = 1 / math.sqrt(128)
    for b in range(4):
        nodes = list(rows[b])[:count[b]]
        for h in range(Hkv):
            used = d.used(b, h)
            want = before[b, h].double()
            err = 2.0 ** -23 * want.abs()
            g_want, g_err = torch.zeros(steps, dtype=torch.float64, device="cuda"), torch.zeros(steps, dtype=torch.float64,
                                                                                             device="cuda")
            for at, i in enumerate(nodes):
                for j in range(h * d.G, (h + 1) * d.G):
                    e = float(lse[b, j, i])
                    if math.isinf(e):
                        continue
                    q = d.q[b, j, i].double()
                    for keys, to, bound, where in ((d.cache.k_hi[b, h, used].double(), want, err, used),
                                                   (d.k[b, h, nodes[:at + 1]].double(), g_want, g_err,
                                                    torch.arange(at + 1, device="cuda"))):
                        s = scale * (keys @ q)
                        w = torch.exp(s - e)
                        # products summed in fp32, the exponential's argument rounded, ex2's own error, sums of <= 72
                        E = scale * 2.0 ** -19 * (keys.abs() @ q.abs()) + 2.0 ** -22 * (s.abs() + abs(e))
                        to.index_add_(0, where, w)
                        bound.index_add_(0, where, w * (torch.expm1(2 * E) + 2.0 ** -17))
            near(d.cache.acc[b, h], want, err + 2.0 ** -23 * want.abs(), f"acc {b} {h}")
            near(gained[b, h], g_want, g_err, f"gained {b} {h}")
            other = torch.ones(d.shape.hi_stride, dtype=torch.bool, device="cuda")
            other[used] = False
            assert torch.equal(d.cache.acc[b, h][other], before[b, h][other])  # nothing else is written


def commit_reference(d, rows, gained, first):
    """The state after a commit, request by request and head by head: a sort, and the oracle's quantizer."""
    s, c = d.shape, d.cache
    st = {x: getattr(c, x).cpu().clone() for x in ARRAYS}
    free = None if d.free is None else d.free.cpu()
    spare = 0 if free is None else 1
    n_hi, n_lo, nxt = list(d.n_hi), list(d.n_lo), list(first)
    k_new, v_new = d.k.cpu(), d.v.cpu()
    bal = None if c.balancer is None else c.balancer.cpu()
    old = {x: st[x].clone() for x in ARRAYS}
    for b, path in enumerate(rows):
        path = list(path) if n_hi[b] > 0 else []
        gone = max(0, n_hi[b] - spare + len(path) - (s.hi_cap - spare)) if path else 0
        if s.bits and n_lo[b] + gone > s.lo_cap:
            continue
        for h in range(s.heads_kv):
            entries = [(float(old["acc"][b, h, t]) + 0.0, int(old["hi_tok"][b, h, t]), t, None) for t in range(n_hi[b])
                       if free is None or t != int(free[b, h])]
            entries += [(float(gained[b, h, i]) + 0.0, first[b] + i, s.hi_cap + i, i) for i in range(len(path))]
            leave = sorted(entries, key=lambda e: e[:3])[:gone]
            for j, (_, tok, t, i) in enumerate(leave):
                if not s.bits:
                    continue
                row = n_lo[b] + j
                for kind in "kv":
                    x = (old[kind + "_hi"][b, h, t] if i is None else (k_new if kind == "k" else v_new)[b, h, path[i]]).float()
                    if kind == "k" and bal is not None:
                        x = x * bal[h]
                    codes, params = oracle.quantize_row(x.numpy(), s.bits, s.group)
                    st[kind + "_codes"][b, h, row] = torch.from_numpy(codes)
                    st[kind + "_params"][b, h, row] = torch.from_numpy(params.view(np.float16))
                st["lo_tok"][b, h, row] = tok
            places = [e[2] for e in leave if e[3] is None] + list(range(n_hi[b], s.hi_cap))
            demoted = {e[3] for e in leave}
            for place, i in zip(places, [i for i in range(len(path)) if i not in demoted]):
                st["k_hi"][b, h, place], st["v_hi"][b, h, place] = k_new[b, h, path[i]], v_new[b, h, path[i]]
                st["hi_tok"][b, h, place], st["acc"][b, h, place] = first[b] + i, gained[b, h, i]
        n_hi[b] += len(path) - gone
        n_lo[b] += gone if s.bits else 0
        nxt[b] += len(path)
    return st, n_hi, n_lo, nxt


def same(a, b, what):
    if a.dtype.is_floating_point:  # bit for bit, NaN included
        a, b = (x.contiguous().view({2: torch.int16, 4: torch.int32}[x.element_size()]) for x in (a, b))
    assert torch.equal(a.cpu(), b.cpu()), what


def check_commit(d, rows, gained, first, steps, fails=False, in_place=False):
    want, n_hi, n_lo, nxt = commit_reference(d, rows, gained, first)
    hi_out, lo_out, next_out = d.dev([-9] * len(rows)), d.dev([-9] * len(rows)), d.dev(first)
    out = pkg.Lengths(hi_out, lo_out)
    if in_place:
        hi_out, lo_out = d.dev(d.n_hi), d.dev(d.n_lo)
        d.lens = out = pkg.Lengths(hi_out, lo_out, d.free)
    ws = torch.zeros(pkg.mikv_commit_workspace_bytes(d.shape, steps), dtype=torch.uint8, device="cuda")
    pkg.mikv_commit_path(d.cache, path_tensor(rows, steps), d.k, d.v, gained.cuda(), next_out, ws, lens=d.lens, lens_out=out,
                         next=next_out)
    if fails:
        with pytest.raises(pkg.MikvError):
            pkg.mikv_workspace_check(ws)
    else:
        pkg.mikv_workspace_check(ws)
    for x in ARRAYS:
        same(getattr(d.cache, x), want[x], x)
    assert hi_out.tolist() == n_hi and lo_out.tolist() == n_lo and next_out.tolist() == nxt


@pytest.mark.parametrize("bits,group", [(2, 32), (2, 64), (2, 128), (3, 32), (3, 64), (3, 128), (4, 32), (4, 64), (4, 128),
                                        (0, 32)])
@pytest.mark.parametrize("in_place", [False, True])
def test_commit(bits, group, in_place):
    """Full requests, growing ones, empty paths, freed requests; scores above, among and below those that are there."""
    hi, lo, steps = 40, 64, 9
    d = drafts(bits + group, B=6, hi=hi, lo=lo, bits=bits, group=group, n_hi=[hi, 3, hi, 0, hi - 4, 1],
               n_lo=[30, 0, 64, 0, 1, 5] if bits else None)
    rows = [[0, 1, 2, 3, 4], [0, 1, 2], [], [0, 1], [0, 1, 2, 3, 4, 5, 6, 7, 8], [0]]
    gained = torch.exp(2 * torch.randn(6, 2, steps, generator=gen(3, "cpu"))) * 0.2
    check_commit(d, rows, gained, [500, 0, 300, 7, 40, 6], steps, in_place=in_place)


@pytest.mark.parametrize("hi", [1, 2, 300])
def test_commit_small_budgets_and_ties(hi):
    """A budget of nothing (every token is demoted), of one; equal scores, zeros of both signs, everything tied."""
    for free in (True, False):
        d = drafts(hi, hi=hi, lo=64, n_lo=[0, 3, 10, 48], free=free)
        d.cache.acc.copy_(torch.randint(0, 2, d.cache.acc.shape, generator=gen(4), device="cuda").float())
        d.cache.acc[:, :, ::3] = -0.0
        gained = torch.randint(0, 2, (4, 2, 9), generator=gen(5, "cpu")).float()
        rows = [[0, 1, 2, 3, 4, 5, 6, 7, 8], [0], [0, 1], [0, 1, 2]]
        check_commit(d, rows, gained, [hi + x for x in (1, 4, 12, 60)], 9)


def test_commit_without_room():
    """A request whose retained rows are full keeps its state; the others go on; the workspace says so."""
    d = drafts(6, hi=30, lo=32, n_lo=[31, 32, 30, 0])
    gained = torch.rand(4, 2, 3, generator=gen(6, "cpu"))
    check_commit(d, [[0, 1], [0], [0, 1], [0, 1, 2]], gained, [90, 90, 90, 30], 3, fails=True)


def test_commit_where_no_slot_is_free():
    """A KV head whose free slot is no slot in use is left alone, and the workspace says so."""
    d = drafts(7, B=1, hi=30, lo=32, n_lo=[4])
    d.free[0, 1] = 30
    old = {x: getattr(d.cache, x)[0, 1].clone() for x in ARRAYS}
    ws = torch.zeros(pkg.mikv_commit_workspace_bytes(d.shape, 2), dtype=torch.uint8, device="cuda")
    gained = torch.rand(1, 2, 2, generator=gen(7), device="cuda")
    pkg.mikv_commit_path(d.cache, path_tensor([[0, 1]], 2), d.k, d.v, gained, d.dev([40]), ws, lens=d.lens)
    with pytest.raises(pkg.MikvError):
        pkg.mikv_workspace_check(ws)
    for x in ARRAYS:
        same(getattr(d.cache, x)[0, 1], old[x], x)


def test_commit_of_a_long_path_and_many_slots():
    """128 accepted tokens; more slots than a block has threads by far."""
    d = Drafts(8, 1, 2, 2, 128, 9001, 208, 4, 32, parents=[[i - 1 for i in range(128)]], n_lo=[50])
    gained = torch.exp(torch.randn(1, 2, 128, generator=gen(8, "cpu")))
    check_commit(d, [range(128)], gained, [20000], 128)


def random_cache(shape, seed):
    c = pkg.LayerCache(shape)
    g = gen(seed)
    for x in ARRAYS + ("k_hi_params", "v_hi_params"):
        t = getattr(c, x)
        if t is not None:
            t.view(torch.uint8).copy_(torch.randint(0, 256, t.view(torch.uint8).shape, generator=g, device="cuda"))
    return c


COPIES = [dict(bits=2, group=32), dict(bits=3, group=128), dict(bits=4, group=64), dict(bits=0, group=32),
          dict(bits=2, group=64, hi_bits=8), dict(bits=3, group=32, hi_bits=2), dict(bits=3, group=64, k_channel_group=64)]


@pytest.mark.parametrize("kw", COPIES, ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
@pytest.mark.parametrize("within", [True, False])
def test_copies(kw, within):
    """Requests of several lengths, to rows of the same cache and of one with more room: what they hold is copied bit for
    bit, nothing else is touched."""
    kch = kw.get("k_channel_group", 0)
    hi, lo = 75, 192
    s = pkg.Shape(6, 4, 2, hi_cap=hi, lo_cap=lo, **kw)
    t = s if within else pkg.Shape(7, 8, 2, hi_cap=hi if kch else hi + 30, lo_cap=lo + 320, **kw)
    a = random_cache(s, 1)
    b = a if within else random_cache(t, 2)
    n_hi, n_lo = [hi, 1, 0, 33, 20, 70], [lo, 0, 1, 130, 191, 64] if s.bits else [0] * 6
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    slots = torch.arange(12, dtype=torch.int32, device="cuda").view(6, 2)
    lens = pkg.Lengths(dev(n_hi), dev(n_lo), slots)
    to = lens if within else pkg.Lengths(dev([-1] * 7), dev([-1] * 7), torch.full((7, 2), -1, dtype=torch.int32, device="cuda"))
    pairs = [(0, 2), (3, 1), (0, 4)] if within else [(0, 6), (5, 0), (3, 3), (2, 1), (1, 2), (4, 5), (0, 4)]
    want = {x: None if getattr(b, x) is None else getattr(b, x).clone() for x in ARRAYS + ("k_hi_params", "v_hi_params")}
    want_len = [x.clone() for x in (to.n_hi, to.n_lo, to.slots)]
    for i, j in pairs:
        kept = n_lo[i] // 64 * 64 if kch else n_lo[i]
        for x in want:
            if want[x] is None:
                continue
            src, dst = getattr(a, x)[i], want[x][j]
            if x in ("k_hi", "v_hi", "hi_tok", "acc", "k_hi_params", "v_hi_params"):
                dst[:, :n_hi[i]] = src[:, :n_hi[i]]
                if kch:
                    dst[:, hi:hi + n_lo[i] - kept] = src[:, hi:hi + n_lo[i] - kept]
            else:
                rows = kept // 64 if kch and x == "k_params" else kept
                dst[:, :rows] = src[:, :rows]
        for w, v in zip(want_len, (dev(n_hi), dev(n_lo), slots.clone())):
            w[j] = v[i]
    pkg.mikv_copy_requests(a, b, pairs, lens=lens, to_lens=to)
    for x in want:
        if want[x] is not None:
            same(getattr(b, x), want[x], x)
    for got, w in zip((to.n_hi, to.n_lo, to.slots), want_len):
        assert torch.equal(got, w)


def test_many_copies_and_none():
    """More pairs than one launch takes; no pairs at all; lengths left out."""
    s = pkg.Shape(1, 1, 1, 2, 32, 20, 32)
    t = pkg.Shape(700, 1, 1, 2, 32, 20, 32)
    a, b = random_cache(s, 3), random_cache(t, 4)
    old = b.k_hi.clone()
    pkg.mikv_copy_requests(a, b, [])
    assert torch.equal(b.k_hi.view(torch.int16), old.view(torch.int16))
    pkg.mikv_copy_requests(a, b, [(0, i) for i in range(700)], lens=pkg.Lengths(n_lo=32))
    for x in ARRAYS:
        got, src = getattr(b, x), getattr(a, x)
        rows = 20 if x in ("k_hi", "v_hi", "hi_tok", "acc") else 32
        same(got[:, :, :rows], src[:, :, :rows].expand(700, *src.shape[1:2], rows, *src.shape[3:]), x)


def test_copies_of_uncounted_requests():
    """A source whose lengths have no arrays: the target's take its slots and rows in use, its free slots are left alone."""
    s, t = pkg.Shape(2, 2, 2, 2, 32, 20, 32), pkg.Shape(3, 2, 2, 2, 32, 33, 48)
    a, b = random_cache(s, 5), random_cache(t, 6)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    to = pkg.Lengths(dev([7, 8, 9]), dev([1, 2, 3]), torch.full((3, 2), 5, dtype=torch.int32, device="cuda"))
    with pytest.raises(pkg.MikvError) as e:
        pkg.mikv_copy_requests(a, b, [(0, 2)], lens=pkg.Lengths(n_lo=30), to_lens=to)
    assert e.value.status == "MIKV_ERR_ARG" and to.n_hi.tolist() == [7, 8, 9] and to.slots.tolist() == [[5, 5]] * 3
    to.slots = None
    old = {x: getattr(b, x).clone() for x in ARRAYS}
    pkg.mikv_copy_requests(a, b, [(0, 2)], lens=pkg.Lengths(n_lo=30), to_lens=to)
    assert to.n_hi.tolist() == [7, 8, 20] and to.n_lo.tolist() == [1, 2, 30]
    for x in ARRAYS:
        rows = 20 if x in ("k_hi", "v_hi", "hi_tok", "acc") else 30
        old[x][2, :, :rows] = getattr(a, x)[0, :, :rows]
        same(getattr(b, x), old[x], x)


def test_drafts_run_together():
    """A prompt's cache, then trees, accepted paths, a fork, trees again: every tree is attended over what the caches hold
    then, every token is somewhere, in bf16 as it came or quantized from that, and the lengths add up."""
    B, Hq, Hkv, T, N, steps = 4, 8, 2, 200, 12, 4
    g = gen(20)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)  # noqa: E731
    shape = pkg.shape_for_context(B, Hq, Hkv, 4, 32, T, 0.2, 40)
    k0, v0, q0 = rand(B, Hkv, T, 128), rand(B, Hkv, T, 128), rand(B, Hq, T, 128)
    table = pkg.RotaryTable()
    pkg.mikv_rotary(table, q0, k0)
    own = pkg.layer.MixedPrecisionLayer.from_prefill(shape, k0, v0, None, q0)
    layer = DraftedLayer.of(own, table, N, steps)
    keys = [{t: (k0[b, :, t], v0[b, :, t]) for t in range(T)} for b in range(B)]
    with pytest.raises(ValueError):
        layer.commit(path_tensor([[0]] * B, steps))
    for step in range(5):
        if step == 3:
            layer.fork([(0, 2)])
            keys[2] = dict(keys[0])
        q, k, v = (rand(B, N, H, 128).transpose(1, 2) for H in (Hq, Hkv, Hkv))
        parents = torch.tensor([[-1, 0, 1, 2, 3, 0, 5, 6, 1, 8, -1, 10]] * B, dtype=torch.int32, device="cuda")
        parents[1, 9:] = -2
        out = torch.empty(B, N, Hq, 128, dtype=BF, device="cuda").transpose(1, 2)
        raw_k = k.clone()
        layer.attend(q, k, v, parents, out)
        tokens = layer.tokens.tolist()
        d = Drafts.__new__(Drafts)
        d.shape, d.cache, d.N, d.G, d.free = shape, layer.cache, N, Hq // Hkv, layer.lens.slots
        d.n_hi, d.n_lo, d.q, d.k, d.v = layer.lens.n_hi.tolist(), layer.lens.n_lo.tolist(), q, k, v
        from _tree_ref import see_brute
        d.see = see_brute(parents.tolist())
        check(d, out, layer.lse, heads=(0, 7))
        pos = torch.tensor([[t + max(len(x) - 1, 0) for x in d.see[b]] for b, t in enumerate(tokens)], dtype=torch.int32,
                           device="cuda")
        pkg.mikv_rotary(table, raw_k, positions=pos)
        assert torch.equal(raw_k, k)
        rows = [[0, 1, 2, 3], [0, 5], [], [0, 1, 8, 9]]
        if step == 4:
            rows[2] = [10]
        layer.commit(path_tensor(rows, steps))
        layer.check()
        for b, path in enumerate(rows):
            for i, node in enumerate(path):
                keys[b][tokens[b] + i] = (k[b, :, node].clone(), v[b, :, node].clone())
            assert int(layer.tokens[b]) == tokens[b] + len(path) == len(keys[b])
            n_hi, n_lo = int(layer.lens.n_hi[b]), int(layer.lens.n_lo[b])
            assert n_hi - 1 + n_lo == len(keys[b])
            for h in range(Hkv):
                slots = [s for s in range(n_hi) if s != int(layer.lens.slots[b, h])]
                hi = layer.cache.hi_tok[b, h, slots].tolist()
                lo = layer.cache.lo_tok[b, h, :n_lo].tolist()
                assert sorted(hi + lo) == sorted(keys[b])
                for s, t in zip(slots, hi):
                    assert torch.equal(layer.cache.k_hi[b, h, s], keys[b][t][0][h])
                    assert torch.equal(layer.cache.v_hi[b, h, s], keys[b][t][1][h])
                got = values_of(layer.cache.v_codes[b, h, :n_lo], layer.cache.v_params[b, h, :n_lo], 4)
                want = torch.stack([keys[b][t][1][h] for t in lo]).double()
                alpha = layer.cache.v_params[b, h, :n_lo, :, 0].double().repeat_interleave(32, 1)
                assert bool(((got - want).abs() <= 0.5 * alpha * (1 + 2.0 ** -10)).all())


def test_commit_refuses_when_the_cache_is_full():
    shape = pkg.Shape(1, 2, 2, 2, 32, 4, 16)
    layer = DraftedLayer(pkg.LayerCache(shape), pkg.RotaryTable(), 3, 3, *(torch.tensor(x, dtype=torch.int32, device="cuda")
                         for x in ([4], [14], [[3, 3]], [17])))
    q = torch.zeros(1, 2, 3, 128, dtype=BF, device="cuda")
    parents = torch.tensor([[-1, 0, 1]], dtype=torch.int32, device="cuda")
    layer.attend(q, q.clone(), q.clone(), parents, torch.empty_like(q))
    with pytest.raises(pkg.MikvError) as e:
        layer.commit(path_tensor([[0]], 3))
    assert e.value.status == "MIKV_ERR_CAPACITY" and layer.tokens.tolist() == [17]


def test_a_step_in_a_graph():
    """Tree, importance and commit captured once, replayed for several steps, against the same steps call by call."""
    def make():
        d = drafts(30, hi=40, lo=64, n_hi=[40, 10, 40, 39], n_lo=[3, 0, 5, 20])
        layer = DraftedLayer(d.cache, pkg.RotaryTable(), d.N, 4, d.dev(d.n_hi), d.dev(d.n_lo), d.free, d.dev([42, 9, 44, 58]), 20)
        return d, layer
    path = path_tensor([[0, 1], [0], [0, 1, 2], []], 4)
    results = []
    for graphed in (False, True):
        d, layer = make()
        q0, k0 = d.q.clone(), d.k.clone()
        q, k = d.q, d.k
        out = torch.empty_like(q0)

        def step():
            q.copy_(q0), k.copy_(k0)
            layer.attend(q, k, d.v, d.parents, out)
            layer.commit(path)
        if graphed:
            saved = {x: getattr(d.cache, x).clone() for x in ARRAYS}
            lens = [x.clone() for x in (layer.lens.n_hi, layer.lens.n_lo, layer.tokens)]
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for x in ARRAYS:
                same(getattr(d.cache, x), saved[x], x)  # capturing runs nothing
            assert all(torch.equal(x, y) for x, y in zip(lens, (layer.lens.n_hi, layer.lens.n_lo, layer.tokens)))
            for _ in range(4):
                g.replay()
        else:
            for _ in range(4):
                step()
        layer.check()
        results.append([getattr(d.cache, x).clone() for x in ARRAYS] + [out, layer.lse, layer.lens.n_hi, layer.lens.n_lo,
                                                                         layer.tokens])
    for a, b in zip(*results):
        same(a, b, "graph")


def full_soon(n_lo, steps=3):
    """A layer of one request whose every accepted token demotes one, 16 retained rows, and a chain for it."""
    d = drafts(31, B=1, N=3, hi=4, lo=16, n_lo=[n_lo])
    layer = DraftedLayer(d.cache, pkg.RotaryTable(), 3, steps, d.dev(d.n_hi), d.dev(d.n_lo), d.free, d.dev([3 + n_lo]), n_lo)
    out = torch.empty_like(d.q)
    return d, layer, lambda: layer.attend(d.q, d.k, d.v, d.parents, out)


def test_commits_after_replays_refuse_before_anything_changes():
    """Replayed steps fill the cache; the next commit, call by call, is refused on the host."""
    d, layer, attend = full_soon(4)
    path = path_tensor([[0, 1, 2]], 3)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend()
        layer.commit(path)
    for _ in range(3):
        g.replay()
    attend()
    layer.commit(path)  # the last that has room
    layer.check()
    assert layer.lens.n_lo.tolist() == [16] and layer.tokens.tolist() == [19]
    attend()
    old = {x: getattr(d.cache, x).clone() for x in ARRAYS}
    with pytest.raises(pkg.MikvError) as e:
        layer.commit(path)
    assert e.value.status == "MIKV_ERR_CAPACITY"
    for x in ARRAYS:
        same(getattr(d.cache, x), old[x], x)
    assert layer.lens.n_lo.tolist() == [16] and layer.tokens.tolist() == [19]
    layer.check()  # no kernel refused anything


def test_a_captured_commit_without_the_room_is_refused():
    """As an error of the library's own, with the capture left whole."""
    d, layer, attend = full_soon(14)
    path = path_tensor([[0]], 3)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend()
        with pytest.raises(pkg.MikvError) as e:
            layer.commit(path)
    assert e.value.status == "MIKV_ERR_CAPACITY" and layer.lens.n_lo.tolist() == [14]
    g.replay()
    layer.check()


def test_forks_of_nothing_keep_the_tree():
    """And forks of a request drop it: a commit then asks for another."""
    d = drafts(32, hi=40, lo=64, n_hi=[40, 10, 40, 39], n_lo=[3, 0, 5, 20])
    layer = DraftedLayer(d.cache, pkg.RotaryTable(), d.N, 4, d.dev(d.n_hi), d.dev(d.n_lo), d.free, d.dev([42, 9, 44, 58]))
    layer.attend(d.q, d.k, d.v, d.parents, torch.empty_like(d.q))
    layer.fork([])
    layer.commit(path_tensor([[0]] * 4, 4))
    assert layer.tokens.tolist() == [43, 10, 45, 59]
    layer.attend(d.q, d.k, d.v, d.parents, torch.empty_like(d.q))
    layer.fork([(0, 1)])
    with pytest.raises(ValueError):
        layer.commit(path_tensor([[0]] * 4, 4))
    assert layer.tokens.tolist() == [43, 43, 45, 59]
    layer.check()


def test_trees_that_are_refused_turn_nothing():
    """Operands that the attention does not take, though the rotary positions would: q and k are as they were, and the same
    tree may come again."""
    d = drafts(33, hi=40, lo=64, n_hi=[40, 10, 40, 39], n_lo=[3, 0, 5, 20])
    layer = DraftedLayer(d.cache, pkg.RotaryTable(), d.N, 4, d.dev(d.n_hi), d.dev(d.n_lo), d.free, d.dev([42, 9, 44, 58]))
    q0, k0, out = d.q.clone(), d.k.clone(), torch.empty_like(d.q)
    room = torch.empty(d.v.numel() + 8, dtype=BF, device="cuda")
    odd = room[1:1 + d.v.numel()].view(d.v.transpose(1, 2).shape).transpose(1, 2)  # rows off a 16-byte boundary
    assert odd.data_ptr() % 16
    pitch = torch.empty(4, d.N, 2, 132, dtype=BF, device="cuda")[..., :128].transpose(1, 2)  # and at strides of 264 bytes
    for v, o in ((odd, out), (pitch, out), (d.v.float(), out), (d.v[:, :, 1:], out), (d.v, out.half()), (d.v, out[:, 1:]),
                 (d.v[:1].expand(4, -1, -1, -1), out), (d.v.cpu(), out)):
        with pytest.raises(ValueError):
            layer.attend(d.q, d.k, v, d.parents, o)
        same(d.q, q0, "q"), same(d.k, k0, "k")
        assert layer.drafted is None
    layer.attend(d.q, d.k, d.v, d.parents, out.float())
    layer.check()
