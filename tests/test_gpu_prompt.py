"""Prompt attention and shared-prefix attention on the GPU against the definition in 64 bits (bounds of
_attn_ref.attention), at the sizes and masks where they can go wrong."""
import math

import pytest
import torch

import paper_2402_18096_gb300 as pkg
import _attn_ref as ref

pytestmark = pytest.mark.gpu

BF, FH, F32 = torch.bfloat16, torch.float16, torch.float32
SCALE = 1 / math.sqrt(128)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(g, shape, dtype, token_major=False, big=False):
    B, H, T, d = shape
    x = torch.randn(B, T, H, d, generator=g, device="cuda") if token_major else torch.randn(shape, generator=g,
                                                                                             device="cuda")
    if big:
        x[..., 5] *= 5
        x[..., 69] *= 5
    x = x.to(dtype)
    return x.transpose(1, 2) if token_major else x


def slopes_of(H):
    return torch.tensor([2.0 ** (-8 * (h + 1) / H) for h in range(H)], device="cuda")


def near(got, want, bound, what):
    g = got.double()
    same = torch.isfinite(want) == torch.isfinite(g)
    assert bool(same.all()), f"{what}: finite where it should not be, or the reverse"
    fin = torch.isfinite(want)
    assert bool((g[~fin] == want[~fin]).all()), what
    err = (g - want).abs()[fin]
    b = bound.expand_as(want)[fin]
    assert bool((err <= b).all()), f"{what}: {float((err / b.clamp(min=1e-300)).max()):.3f} of the bound"


def check_prompt(q, k, v, out, lse, spans, scale=SCALE, cap=0.0, slopes=None, q_start=0, heads=None):
    """spans [B, tq, 2] int (any device); heads: query heads to check (all)."""
    B, Hq, tq, _ = q.shape
    Hkv, tk = k.shape[1], k.shape[2]
    spans = spans.cuda()
    pos = q_start + torch.arange(tq, device="cuda")
    for b in range(B):
        mask = ref.span_mask(spans[b, :, 0], spans[b, :, 1], tk)
        for h in heads or range(Hq):
            kv = h // (Hq // Hkv)
            s = None if slopes is None else slopes[h].expand(tq)
            o, e, ob, eb = ref.attention(q[b, h], k[b, kv], v[b, kv], mask, scale, cap, s, pos, out.dtype)
            near(out[b, h], o, ob, f"out b{b} h{h}")
            if lse is not None:
                near(lse[b, h], e, eb, f"lse b{b} h{h}")


def prompt(q, k, v, out_dtype=None, major=False, ws=None, **kw):
    B, Hq, tq, d = q.shape
    dt = out_dtype or q.dtype
    out = torch.full((B, tq, Hq, d), math.nan, dtype=dt, device="cuda").transpose(1, 2) if major else \
        torch.full((B, Hq, tq, d), math.nan, dtype=dt, device="cuda")
    lse = torch.full((B, Hq, tq), math.nan, device="cuda")
    ws = torch.zeros(pkg.mikv_prompt_workspace_bytes(q, k), dtype=torch.uint8, device="cuda") if ws is None else ws
    pkg.mikv_prompt_attention(q, k, v, out, ws, lse=lse, **kw)
    pkg.mikv_workspace_check(ws)
    return out, lse


def causal_spans(B, tq, tk, q_start):
    hi = (q_start + 1 + torch.arange(tq)).clamp(0, tk)
    return torch.stack([torch.zeros_like(hi), hi], dim=1).expand(B, tq, 2)


# (B, Hq, Hkv, tq, tk): one token, tiles exactly, one past, one short, ragged, several tiles of queries and keys
SHAPES = [(1, 1, 1, 1, 1), (2, 4, 2, 5, 5), (1, 2, 2, 127, 127), (1, 2, 1, 128, 128), (1, 1, 1, 129, 129),
          (2, 8, 1, 33, 33), (1, 4, 4, 257, 257), (1, 4, 1, 515, 515), (2, 8, 2, 700, 700),
          (1, 2, 2, 3, 640), (3, 8, 1, 1, 1000), (1, 4, 2, 100, 1500), (1, 8, 2, 17, 4099)]


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_causal(shape, dtype):
    B, Hq, Hkv, tq, tk = shape
    g = gen(tq + tk)
    q, k, v = make(g, (B, Hq, tq, 128), dtype), make(g, (B, Hkv, tk, 128), dtype, big=True), make(g, (B, Hkv, tk, 128),
                                                                                              dtype)
    out, lse = prompt(q, k, v)
    check_prompt(q, k, v, out, lse, causal_spans(B, tq, tk, tk - tq), q_start=tk - tq)


@pytest.mark.parametrize("shape", [(2, 8, 2, 300, 300), (1, 2, 1, 130, 1100), (1, 8, 8, 64, 90)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("cap,bias", [(0.0, True), (30.0, False), (5.0, True)])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (FH, F32)])
def test_capped_and_biased(shape, cap, bias, dtype, out_dtype):
    """Caps (5: most scores are bent), a bias by distance on both sides of the query (causal and not)."""
    B, Hq, Hkv, tq, tk = shape
    g = gen(7 * tq + tk)
    q, k, v = (make(g, (B, H, T, 128), dtype, token_major=True, big=big) for H, T, big in
               ((Hq, tq, False), (Hkv, tk, True), (Hkv, tk, False)))
    sl = slopes_of(Hq) if bias else None
    for causal in (True, False):
        out, lse = prompt(q, k, v, out_dtype=out_dtype, major=True, causal=causal, softcap=cap, slopes=sl)
        spans = causal_spans(B, tq, tk, tk - tq) if causal else torch.tensor([0, tk]).expand(B, tq, 2)
        check_prompt(q, k, v, out, lse, spans, cap=cap, slopes=sl, q_start=tk - tq)


def test_spans_against_brute_force():
    docs = torch.tensor([[0, 3, 3, 40, 70], [5, 6, 90, 100, 100]], dtype=torch.int32, device="cuda")
    pre_d = torch.tensor([[1, 0, 20, 999], [1, 2, 3, 4]], dtype=torch.int32, device="cuda")
    pre = torch.tensor([0, 55], dtype=torch.int32, device="cuda")
    klen = torch.tensor([64, 7], dtype=torch.int32, device="cuda")
    for tq, tk, q_start in ((100, 100, 0), (37, 100, 63), (20, 60, -5), (1, 1, 0), (30, 40, 35)):
        for causal in (True, False):
            for d in (None, docs):
                for p in (None, pre if d is None else pre_d):
                    for n in (None, klen):
                        got = torch.empty(2, tq, 2, dtype=torch.int32, device="cuda")
                        pkg.mikv_mask_spans(got, tk, q_start=q_start, causal=causal, docs=d, prefix=p, key_len=n)
                        want = ref.spans_brute(2, tq, tk, q_start, causal, *(None if x is None else x.tolist()
                                                                             for x in (d, p, n)))
                        assert torch.equal(got.cpu(), want), (tq, tk, q_start, causal, d is None, p is None, n is None)


@pytest.mark.parametrize("Hq,Hkv,dtype", [(4, 4, BF), (8, 2, FH), (8, 1, BF)])
def test_documents_prefixes_and_padding(Hq, Hkv, dtype):
    """Packed documents (one of a single token, an empty one, padding behind the last), prefixes seen from both
    sides, key lengths; with a bias. Rows that see nothing give zeros and -inf."""
    B, T = 2, 431
    g = gen(Hq)
    q, k, v = (make(g, (B, H, T, 128), dtype) for H in (Hq, Hkv, Hkv))
    docs = torch.tensor([[0, 130, 131, 131, 300, 420], [2, 50, 51, 200, 390, 431]], dtype=torch.int32, device="cuda")
    pre = torch.tensor([[0, 1, 0, 100, 5], [48, 0, 0, 190, 1]], dtype=torch.int32, device="cuda")
    klen = torch.tensor([431, 260], dtype=torch.int32, device="cuda")
    sl = slopes_of(Hq)
    for kw in (dict(docs=docs), dict(docs=docs, prefix=pre), dict(prefix=pre[:, 3].contiguous()),
               dict(key_len=klen), dict(docs=docs, key_len=klen, causal=False)):
        spans = torch.empty(B, T, 2, dtype=torch.int32, device="cuda")
        pkg.mikv_mask_spans(spans, T, **kw)
        for s in (None, sl):
            out, lse = prompt(q, k, v, spans=spans, slopes=s)
            check_prompt(q, k, v, out, lse, spans, slopes=s)
            empty = spans[..., 0] >= spans[..., 1]
            assert bool((out.transpose(1, 2)[empty] == 0).all())
            assert bool((lse.transpose(1, 2)[empty] == -math.inf).all())


def test_any_spans():
    """Spans that no rule makes: empty, reversed, out of range, single keys, each row another."""
    B, Hq, Hkv, tq, tk = 2, 4, 2, 150, 1000
    g = gen(11)
    q, k, v = make(g, (B, Hq, tq, 128), BF), make(g, (B, Hkv, tk, 128), BF), make(g, (B, Hkv, tk, 128), BF)
    a = torch.randint(-50, tk + 50, (B, tq, 2), generator=g, device="cuda", dtype=torch.int32)
    a[:, ::3, 1] = a[:, ::3, 0] + 1
    out, lse = prompt(q, k, v, spans=a)
    check_prompt(q, k, v, out, lse, a.clamp(0, tk))


@pytest.mark.parametrize("q_start", [-40, -1, 0, 17, 500])
def test_query_start(q_start):
    """Queries before the first key see nothing; queries past the last one see all keys."""
    B, Hq, Hkv, tq, tk = 1, 4, 2, 90, 200
    g = gen(12)
    q, k, v = make(g, (B, Hq, tq, 128), BF), make(g, (B, Hkv, tk, 128), BF), make(g, (B, Hkv, tk, 128), BF)
    sl = slopes_of(Hq)
    out, lse = prompt(q, k, v, q_start=q_start, slopes=sl)
    check_prompt(q, k, v, out, lse, causal_spans(B, tq, tk, q_start), slopes=sl, q_start=q_start)


def test_no_keys():
    q = make(gen(1), (1, 2, 5, 128), BF)
    k = torch.empty(1, 1, 0, 128, dtype=BF, device="cuda")
    out, lse = prompt(q, k, k)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["keys", "values"])
def test_masked_places_hold_anything(bad, where):
    """Infinities and NaN in keys and values that a query does not see leave it alone: behind a key length, in
    another document of the same tile, in the causal future."""
    B, Hq, Hkv, T = 1, 4, 2, 400
    g = gen(13)
    q, k, v = make(g, (B, Hq, T, 128), BF), make(g, (B, Hkv, T, 128), BF), make(g, (B, Hkv, T, 128), BF)
    docs = torch.tensor([[0, 90, 150, 390]], dtype=torch.int32, device="cuda")
    spans = torch.empty(B, T, 2, dtype=torch.int32, device="cuda")
    pkg.mikv_mask_spans(spans, T, docs=docs)
    clean, clean_lse = prompt(q, k, v, spans=spans)
    x = k if where == "keys" else v
    x[:, :, 100:140, 3] = bad  # the middle document
    x[:, :, 395:] = bad        # the padding
    out, lse = prompt(q, k, v, spans=spans)
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[100:150] = False
    assert torch.equal(out[:, :, rows], clean[:, :, rows])
    assert torch.equal(lse[:, :, rows], clean_lse[:, :, rows])
    if where == "values" or math.isnan(bad):  # rows 140 .. 149 see all of the bad ones
        assert not bool(torch.isfinite(out[:, :, 140:150, 3]).any())
    # causal: rows before the first bad key
    out, lse = prompt(q, k, v)
    clean2, _ = prompt(q, torch.where(torch.isfinite(k), k, 0), torch.where(torch.isfinite(v), v, 0))
    assert torch.equal(out[:, :, :100], clean2[:, :, :100])


@pytest.mark.parametrize("scale", [1e-3, 3.0])
def test_scales_and_large_scores(scale):
    """Nearly uniform weights, and scores of hundreds whose largest comes late, early or in the middle."""
    B, Hq, Hkv, tq, tk = 1, 2, 1, 140, 1300
    for dtype in (BF, FH):
        g = gen(14)
        q, k, v = make(g, (B, Hq, tq, 128), dtype), make(g, (B, Hkv, tk, 128), dtype), make(g, (B, Hkv, tk, 128), dtype)
        k[:, :, 5] *= 3
        k[:, :, 700] *= 6
        k[:, :, 1299] *= 4
        out, lse = prompt(q, k, v, sm_scale=scale, causal=False)
        check_prompt(q, k, v, out, lse, torch.tensor([0, tk]).expand(B, tq, 2), scale=scale)


def test_equal_keys_and_lowest_scores():
    """All scores equal; all scores at the most negative the type gives (no row becomes empty by it)."""
    tq, tk = 130, 300
    q = torch.ones(1, 1, tq, 128, dtype=BF, device="cuda")
    v = make(gen(15), (1, 1, tk, 128), BF)
    for val in (1.0, -1e30, 0.0):
        k = torch.full((1, 1, tk, 128), val, dtype=BF, device="cuda")
        out, lse = prompt(q, k, v, causal=False)
        check_prompt(q, k, v, out, lse, torch.tensor([0, tk]).expand(1, tq, 2))


def test_shared_keys_with_zero_strides():
    """k, v expanded over the batch and over the KV heads (zero strides), as they are."""
    g = gen(16)
    q = make(g, (3, 4, 77, 128), BF)
    k1, v1 = make(g, (1, 1, 200, 128), BF), make(g, (1, 1, 200, 128), BF)
    k, v = k1.expand(3, 2, 200, 128), v1.expand(3, 2, 200, 128)
    out, lse = prompt(q, k, v)
    check_prompt(q, k, v, out, lse, causal_spans(3, 77, 200, 123), q_start=123)


def test_views_of_packed_projection():
    """q, k and v as views of one [B, T, Hq + 2 Hkv, 128] projection; the output into a wider buffer."""
    B, Hq, Hkv, T = 2, 8, 2, 260
    p = make(gen(17), (B, T, Hq + 2 * Hkv, 128), BF)
    q, k, v = (p[:, :, a:b].transpose(1, 2) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    wide = torch.full((B, T, Hq + 3, 128), 7.0, dtype=BF, device="cuda")
    out = wide[:, :, 1:Hq + 1].transpose(1, 2)
    ws = torch.zeros(pkg.mikv_prompt_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    pkg.mikv_prompt_attention(q, k, v, out, ws)
    check_prompt(q, k, v, out, None, causal_spans(B, T, T, 0))
    assert bool((wide[:, :, 0] == 7).all()) and bool((wide[:, :, Hq + 1:] == 7).all())


def test_offsets_past_32_bits():
    """Keys, values, queries and outputs whose rows lie more than 2^31 elements apart."""
    g = gen(18)
    far = 2 ** 31 + 2 ** 20
    buf = torch.zeros(far + 400 * 128, dtype=BF, device="cuda")
    obuf = torch.zeros(far + 400 * 128, dtype=BF, device="cuda")

    def at(b, off):
        return torch.as_strided(b, (2, 1, 100, 128), (far, 100 * 128, 128, 1), off * 12800)

    q, k, v = at(buf, 0), at(buf, 1), at(buf, 2)
    for x in (q, k, v):
        x.copy_(make(g, (2, 1, 100, 128), BF))
    out = at(obuf, 0)
    ws = torch.zeros(pkg.mikv_prompt_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    pkg.mikv_prompt_attention(q, k, v, out, ws)
    check_prompt(q, k, v, out, None, causal_spans(2, 100, 100, 0))


def test_long_prompt_sampled_heads():
    B, Hq, Hkv, T = 1, 8, 2, 5000
    g = gen(19)
    q, k, v = make(g, (B, Hq, T, 128), BF), make(g, (B, Hkv, T, 128), BF, big=True), make(g, (B, Hkv, T, 128), BF)
    out, lse = prompt(q, k, v)
    check_prompt(q, k, v, out, lse, causal_spans(B, T, T, 0), heads=[0, 5])


def test_repeat_and_other_stream_give_the_same_bits():
    g = gen(20)
    q, k, v = make(g, (2, 8, 333, 128), BF), make(g, (2, 2, 2000, 128), BF), make(g, (2, 2, 2000, 128), BF)
    a, la = prompt(q, k, v)
    b, lb = prompt(q, k, v)
    assert torch.equal(a, b) and torch.equal(la, lb)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c, lc = prompt(q, k, v)
    side.synchronize()
    assert torch.equal(a, c) and torch.equal(la, lc)


def test_in_a_cuda_graph():
    g = gen(21)
    q, k, v = make(g, (1, 4, 3, 128), BF), make(g, (1, 2, 900, 128), BF), make(g, (1, 2, 900, 128), BF)
    want, _ = prompt(q, k, v)
    out = torch.empty_like(q)
    ws = torch.zeros(pkg.mikv_prompt_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.mikv_prompt_attention(q, k, v, out, ws)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


# ------------------------------------------------------------------ shared prefixes

def prefix(q, k, v, out_dtype=None, **kw):
    B, Hq, d = q.shape
    out = torch.full((B, Hq, d), math.nan, dtype=out_dtype or q.dtype, device="cuda")
    ml = torch.full((B, Hq, 2), math.nan, device="cuda")
    ws = torch.zeros(pkg.mikv_prefix_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    pkg.mikv_prefix_attention(q, k, v, out, ws, ml=ml, **kw)
    pkg.mikv_workspace_check(ws)
    return out, ml


def check_prefix(q, k, v, out, ml, lens=None, q_pos=None, cap=0.0, slopes=None, own_out=None, own_ml=None):
    B, Hq, d = q.shape
    n, Hkv, P = k.shape[:3]
    per, G = B // n, Hq // Hkv
    for x in range(n):
        L = P if lens is None else int(lens[x])
        rows = slice(x * per, (x + 1) * per)
        pos = (torch.full((per,), L, device="cuda") if q_pos is None else q_pos[rows]).repeat_interleave(G)
        mask = (torch.arange(P, device="cuda") < L).expand(per * G, P)
        for h in range(Hkv):
            hs = slice(h * G, (h + 1) * G)
            s = None if slopes is None else slopes[hs].repeat(per)
            o, e, ob, eb = ref.attention(q[rows, hs].reshape(-1, d), k[x, h], v[x, h], mask, SCALE, cap, s, pos,
                                         out.dtype)
            if own_out is not None:
                o, e, ob, eb = ref.join(o, e, ob, eb, own_out[rows, hs].reshape(-1, d), own_ml[rows, hs].reshape(-1, 2),
                                        out.dtype)
            near(out[rows, hs].reshape(-1, d), o, ob, f"out group {x} head {h}")
            near(ml[rows, hs, 0].reshape(-1), e, eb, f"lse group {x} head {h}")
            assert torch.equal(ml[rows, hs, 1].reshape(-1), (e != -math.inf).float())


# (B, groups, Hq, Hkv, P): one request, a group's rows just at and over one tile, many, each its own
PREFIX = [(1, 1, 1, 1, 1), (1, 1, 32, 32, 511), (1, 1, 8, 1, 5000), (32, 1, 8, 2, 1000), (33, 1, 4, 1, 700),
          (16, 1, 8, 1, 129), (17, 1, 8, 1, 128), (65, 1, 8, 2, 300), (150, 1, 8, 4, 2100), (6, 3, 8, 2, 640),
          (5, 5, 4, 4, 1030), (40, 2, 16, 2, 257)]


@pytest.mark.parametrize("dtype", [BF, FH])
@pytest.mark.parametrize("shape", PREFIX, ids=lambda s: "x".join(map(str, s)))
def test_prefix(shape, dtype):
    B, n, Hq, Hkv, P = shape
    g = gen(B + P)
    q = torch.randn(B, Hq, 128, generator=g, device="cuda").to(dtype)
    k, v = make(g, (n, Hkv, P, 128), dtype, big=True), make(g, (n, Hkv, P, 128), dtype, token_major=True)
    out, ml = prefix(q, k, v)
    check_prefix(q, k, v, out, ml)


@pytest.mark.parametrize("cap,bias,joined,out_dtype", [(0.0, True, False, BF), (30.0, False, True, BF),
                                                      (4.0, True, True, F32)])
@pytest.mark.parametrize("shape", [(12, 4, 8, 2, 900), (40, 1, 8, 2, 333), (3, 3, 2, 2, 2000)],
                         ids=lambda s: "x".join(map(str, s)))
def test_prefix_ragged_capped_biased_joined(shape, cap, bias, joined, out_dtype):
    """Prefixes of other lengths (none at all among them) with garbage behind their ends, own positions, a join with
    what another cache gave (one request's own part empty)."""
    B, n, Hq, Hkv, P = shape
    g = gen(B * P)
    q = torch.randn(B, Hq, 128, generator=g, device="cuda").to(BF)
    k, v = make(g, (n, Hkv, P, 128), BF), make(g, (n, Hkv, P, 128), BF)
    lens = torch.tensor([P, 0, 1, P - 130][:n], dtype=torch.int32, device="cuda")
    for x in range(n):
        k[x, :, int(lens[x]):] = math.nan
        v[x, :, int(lens[x]):] = math.inf
    q_pos = (P + torch.randint(0, 50, (B,), generator=g, device="cuda")).to(torch.int32)
    q_pos[0] = 20  # before the prefix's end: distance on both sides
    sl = slopes_of(Hq) if bias else None
    own_out = own_ml = None
    if joined:
        own_out = torch.randn(B, Hq, 128, generator=g, device="cuda")
        own_ml = torch.stack([torch.randn(B, Hq, generator=g, device="cuda") * 3,
                              1 + 50 * torch.rand(B, Hq, generator=g, device="cuda")], dim=2).contiguous()
        own_ml[-1, :, 0], own_ml[-1, :, 1], own_out[-1] = -math.inf, 0.0, 0.0
    out, ml = prefix(q, k, v, out_dtype=out_dtype, lens=lens, q_pos=q_pos, softcap=cap, slopes=sl, own_out=own_out,
                     own_ml=own_ml)
    check_prefix(q, k, v, out, ml, lens, q_pos, cap, sl, own_out, own_ml)


@pytest.mark.parametrize("n,Hkv,P", [(70, 2, 1500), (33, 4, 700), (150, 1, 300)])
def test_prefix_many_lengths(n, Hkv, P):
    """More sets of keys than a warp has lanes, lengths from nothing to all, several of them empty in a row: every set
    gets its share of the CTAs."""
    g = gen(n)
    lens = torch.randint(0, P + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    lens[::7] = 0
    lens[30:34] = 0
    lens[-1] = P
    q = torch.randn(n, 4 * Hkv, 128, generator=g, device="cuda").to(BF)
    k, v = make(g, (n, Hkv, P, 128), BF), make(g, (n, Hkv, P, 128), BF)
    out, ml = prefix(q, k, v, lens=lens)
    check_prefix(q, k, v, out, ml, lens)
    lens.zero_()
    out, ml = prefix(q, k, v, lens=lens)
    assert bool((out == 0).all()) and bool((ml[..., 1] == 0).all())


@pytest.mark.parametrize("shape", [(1, 8, 2, 64, 9000), (2, 4, 1, 130, 5000), (1, 1, 1, 300, 7000), (1, 4, 4, 20, 3000)],
                         ids=lambda s: "x".join(map(str, s)))
def test_keys_shared_out(shape):
    """Few queries on long keys: the row tiles' keys are cut for many CTAs, at places that masks make ragged (spans,
    causal)."""
    B, Hq, Hkv, tq, tk = shape
    g = gen(tk)
    q, k, v = make(g, (B, Hq, tq, 128), BF), make(g, (B, Hkv, tk, 128), BF), make(g, (B, Hkv, tk, 128), BF)
    sl = slopes_of(Hq)
    out, lse = prompt(q, k, v, slopes=sl)
    check_prompt(q, k, v, out, lse, causal_spans(B, tq, tk, tk - tq), slopes=sl, q_start=tk - tq)
    a = torch.randint(0, tk, (B, tq, 2), generator=g, device="cuda", dtype=torch.int32).sort(dim=2).values.contiguous()
    a[:, ::5] = 0
    out, lse = prompt(q, k, v, spans=a, softcap=20.0)
    check_prompt(q, k, v, out, lse, a, cap=20.0)


def test_bias_at_far_positions():
    """A bias of far queries differs from that of near ones by a constant per row, which the softmax does not see: with
    exact distances the output stays within the near queries' bounds, through masked tiles and unmasked ones."""
    B, Hq, Hkv, tq, tk = 1, 4, 2, 70, 700
    g = gen(23)
    q, k, v = make(g, (B, Hq, tq, 128), BF), make(g, (B, Hkv, tk, 128), BF), make(g, (B, Hkv, tk, 128), BF)
    sl = slopes_of(Hq)
    spans = torch.empty(B, tq, 2, dtype=torch.int32, device="cuda")
    spans[..., 0] = 3
    spans[..., 1] = tk - 5 - torch.arange(tq, device="cuda") % 40
    full = torch.tensor([0, tk], device="cuda").expand(B, tq, 2)
    for q_start in (tk, 2 ** 17, 2 ** 20):
        for s, kw in ((spans, dict(spans=spans)), (full, dict(causal=False))):
            out, _ = prompt(q, k, v, q_start=q_start, slopes=sl, **kw)
            check_prompt(q, k, v, out, None, s, slopes=sl, q_start=tk)


def test_prefix_empty_everywhere():
    q = torch.randn(2, 4, 128, device="cuda").to(BF)
    k = torch.full((1, 2, 64, 128), math.nan, dtype=BF, device="cuda")
    out, ml = prefix(q, k, k, lens=torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert bool((out == 0).all()) and bool((ml[..., 0] == -math.inf).all()) and bool((ml[..., 1] == 0).all())
    k0 = k[:, :, :0]
    out, ml = prefix(q, k0, k0)
    assert bool((out == 0).all()) and bool((ml[..., 1] == 0).all())


def test_prefix_joined_with_the_mixed_cache_is_attention_over_both():
    """Prefix attention joined with mikv_decode_attention over a request's own (all-important, bf16) cache equals
    attention over the concatenation; the joint statistics serve the importance update."""
    B, Hq, Hkv, P, T = 3, 8, 2, 300, 45
    g = gen(30)
    q = torch.randn(B, Hq, 128, generator=g, device="cuda").to(BF)
    kp, vp = make(g, (1, Hkv, P, 128), BF), make(g, (1, Hkv, P, 128), BF)
    ko, vo = make(g, (B, Hkv, T, 128), BF), make(g, (B, Hkv, T, 128), BF)
    shape = pkg.Shape(B, Hq, Hkv, 0, 32, hi_cap=T, lo_cap=0)
    cache = pkg.LayerCache(shape)
    rows = torch.arange(T, dtype=torch.int32, device="cuda").expand(B, Hkv, T).contiguous()
    pkg.mikv_gather_hi(cache, ko, vo, rows)
    own_out, own_ml = torch.empty(B, Hq, 128, device="cuda"), torch.empty(B, Hq, 2, device="cuda")
    logits = torch.empty(B, Hq, shape.hi_stride, device="cuda")
    ws = torch.zeros(pkg.mikv_workspace_bytes(shape, pkg.WS_ATTENTION, 0), dtype=torch.uint8, device="cuda")
    pkg.mikv_decode_attention(cache, 0, q, SCALE, own_out, ws, hi_logits=logits, ml=own_ml)
    out, ml = prefix(q, kp, vp, own_out=own_out, own_ml=own_ml)
    pkg.mikv_update_importance(cache, logits, ml)
    for b in range(B):
        for h in range(Hkv):
            k = torch.cat([kp[0, h], ko[b, h]])
            v = torch.cat([vp[0, h], vo[b, h]])
            rows_q = q[b, h * 4:h * 4 + 4]
            mask = torch.ones(4, P + T, dtype=torch.bool, device="cuda")
            o, e, ob, eb = ref.attention(rows_q, k, v, mask, SCALE, out_dtype=BF)
            vmax = float(v.double().abs().max())
            near(out[b, h * 4:h * 4 + 4], o, ob + 2e-3 * vmax, "joined")  # (the own part's documented bound)
            near(ml[b, h * 4:h * 4 + 4, 0], e, eb + 2.0 ** -16, "lse")
            w = torch.exp(SCALE * rows_q.double() @ ko[b, h].double().T - e[:, None]).sum(dim=0)
            got = cache.acc[b, h, :T].double()
            assert bool(((got - w).abs() <= 1e-4 * w + 1e-9).all())


# ------------------------------------------------------------------ refusals

def test_wrong_arguments_raise():
    q, k = make(gen(1), (1, 4, 8, 128), BF), make(gen(2), (1, 2, 8, 128), BF)
    out = torch.empty_like(q)
    ws = torch.zeros(pkg.mikv_prompt_workspace_bytes(q, k), dtype=torch.uint8, device="cuda")
    ok = (q, k, k, out, ws)
    pkg.mikv_prompt_attention(*ok)
    for args, kw, err in (
            ((q, k.half(), k, out, ws), {}, ValueError),
            ((q, k, k[:, :, :4], out, ws), {}, ValueError),
            ((q, k, k, out[:, :, :4], ws), {}, ValueError),
            ((q, k, k, out.half(), ws), {}, pkg.MikvError),
            ((q, k, k, out, ws[:16]), {}, pkg.MikvError),
            (ok, dict(sm_scale=0.0), pkg.MikvError),
            (ok, dict(sm_scale=math.nan), pkg.MikvError),
            (ok, dict(softcap=-1.0), pkg.MikvError),
            (ok, dict(slopes=torch.zeros(3, device="cuda")), ValueError),
            (ok, dict(spans=torch.zeros(1, 8, 2, dtype=torch.int64, device="cuda")), ValueError),
            (ok, dict(lse=torch.zeros(1, 4, 7, device="cuda")), ValueError)):
        with pytest.raises(err):
            pkg.mikv_prompt_attention(*args, **kw)
    off = torch.zeros(1, 4, 8, 132, dtype=BF, device="cuda")
    with pytest.raises(pkg.MikvError):  # rows of 264 bytes: strides are no multiples of 16 bytes
        pkg.mikv_prompt_attention(off[..., :128], k, k, out, ws)
    q1 = torch.zeros(4, 4, 128, dtype=BF, device="cuda")
    kp = torch.zeros(3, 2, 8, 128, dtype=BF, device="cuda")
    with pytest.raises(pkg.MikvError):  # 4 requests on 3 prefixes
        pkg.mikv_prefix_attention(q1, kp, kp, torch.empty_like(q1), ws)
