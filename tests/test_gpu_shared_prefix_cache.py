"""The own cache of a shared-prefix layer: importance under the softmax over prefix and own tokens, from the prompt on
and over decode steps whose cache holds retained (quantised) tokens beside the prefix."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2402_18096_gb300 as pkg
from paper_2402_18096_gb300.layer import SharedPrefixLayer, workspace
import _attn_ref as ref
from _cases import bits16, logit_bounds, softmax_stat_bounds
from test_gpu_prefill import prefill_rtol

pytestmark = pytest.mark.gpu

SCALE = 1 / math.sqrt(128)


def make(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def given_scores(q, k, lse):
    """fp32 [B, Hkv, T] of the library for own rows q [B, Hq, T, d], k [B, Hkv, T, d] and given log-sum-exps."""
    B, Hq, T, _ = q.shape
    Hkv = k.shape[1]
    shape = pkg.Shape(B, Hq, Hkv, 2, 32, 1, 16)
    out = torch.full((B, Hkv, T), math.nan, device="cuda")
    ws = workspace(pkg.mikv_workspace_bytes(shape, pkg.WS_PREFILL, T))
    pkg.mikv_prefill_scores(shape, q, k, out, ws, lse=lse)
    pkg.mikv_workspace_check(ws)
    return out


def summed_weights(q, k, lse):
    """The same in 64 bits: sum over query heads and queries i >= t of exp(s_it - lse_i)."""
    B, Hq, T, _ = q.shape
    Hkv = k.shape[1]
    past = torch.ones(T, T, dtype=torch.bool, device="cuda").tril()
    out = torch.zeros(B, Hkv, T, dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            s = SCALE * q[b, h].double() @ k[b, kv].double().T
            w = torch.exp(s - lse[b, h].double()[:, None])
            w[torch.isinf(lse[b, h])] = 0  # (a query without a finite sum weighs nothing)
            out[b, kv] += torch.where(past, w, 0.0).sum(dim=0)
    return out


def given_rtol(q, k, lse):
    """prefill_rtol with the given normaliser in place of the kernel's own: it is turned into log2 units by one fp32
    product with a rounded constant, 2^-23 of its size, which is an absolute error of the exponent."""
    size = float(torch.where(torch.isinf(lse), 0.0, lse).abs().max()) * math.log2(math.e)
    return prefill_rtol(bits16(q), bits16(k), q.shape[2], q.shape[1] // k.shape[1]) + 2 * math.log(2) * 2.0 ** -23 * size


@pytest.mark.parametrize("B,Hq,Hkv,T", [(1, 2, 2, 1), (2, 8, 2, 130), (1, 4, 1, 700), (3, 8, 1, 64)])
def test_scores_with_given_normalisers(B, Hq, Hkv, T):
    g = torch.Generator(device="cuda").manual_seed(T)
    q, k = make(g, B, Hq, T, 128), make(g, B, Hkv, T, 128)
    k[..., 5] *= 5
    lse = 4 + 3 * torch.randn(B, Hq, T, generator=g, device="cuda")
    if T > 1:
        lse[0, 0, T // 2] = -math.inf  # a query that saw nothing
        lse[-1, -1, T - 1] = math.inf
    got, want = given_scores(q, k, lse).double(), summed_weights(q, k, lse)
    assert bool(((got - want).abs() <= given_rtol(q, k, lse) * want).all())


def prompts(g, B, Hq, Hkv, P, T, ratio, steps, bits=2, group=32):
    """A layer from random prompts, with its turned queries and keys."""
    table = pkg.RotaryTable()
    q0, k0, v0 = (make(g, 1, h, P, 128) for h in (Hq, Hkv, Hkv))
    q, k, v = (make(g, B, h, T, 128) for h in (Hq, Hkv, Hkv))
    k0 *= 1.5  # the prefix holds most of the weight
    shape = pkg.shape_for_context(B, Hq, Hkv, bits, group, T, ratio, steps)
    out0 = torch.empty(1, Hq, P, 128, dtype=torch.bfloat16, device="cuda")
    out1 = torch.empty(B, Hq, T, 128, dtype=torch.bfloat16, device="cuda")
    layer = SharedPrefixLayer.from_prompts(shape, table, (q0, k0, v0), (q, k, v), out0, out1)
    return layer, table, (k0, v0), (q, k, v)


def joint_lse(q, k0, k):
    """Log of each own query's sum over prefix and own keys, in 64 bits, and the bound on the kernels' value."""
    B, Hq, T, _ = q.shape
    P, G = k0.shape[2], Hq // k.shape[1]
    lse = torch.empty(B, Hq, T, dtype=torch.float64, device="cuda")
    bound = 0.0
    mask = torch.arange(P + T, device="cuda") <= P + torch.arange(T, device="cuda")[:, None]
    for b in range(B):
        for h in range(Hq):
            keys = torch.cat([k0[0, h // G], k[b, h // G]])
            _, lse[b, h], _, eb = ref.attention(q[b, h], keys, keys, mask, SCALE)
            bound = max(bound, float(eb.max()))
    return lse, bound


def test_prompt_importance_is_that_of_the_whole_softmax():
    """The scores that the own cache starts with are sums of weights over prefix and own keys; the kept tokens are the
    largest of them."""
    B, Hq, Hkv, P, T = 2, 8, 2, 700, 150
    layer, _, (k0, _), (q, k, _) = prompts(torch.Generator(device="cuda").manual_seed(5), B, Hq, Hkv, P, T, 0.2, 4)
    lse, bound = joint_lse(q, k0, k)
    want = summed_weights(q, k, lse)
    # (both statistics of a weight are off: the scores' own bound, twice the bound of the log-sum-exp with its margin)
    rtol = given_rtol(q, k, lse) + 2 * math.expm1(2 * bound)
    n = layer.own.shape.hi_cap - 1
    tok = layer.own.cache.hi_tok[:, :, :n].long()
    at = torch.gather(want, 2, tok)
    assert bool(((layer.own.cache.acc[:, :, :n].double() - at).abs() <= rtol * at).all())
    edge = want.sort(dim=2, descending=True).values[:, :, n - 1:n]
    assert bool((at >= edge * (1 - 2 * rtol)).all())


def test_the_prefix_is_not_copied_for_each_request():
    """What from_prompts allocates stays well below the prefix's keys and values once per request."""
    B, Hq, Hkv, P, T = 128, 8, 2, 2048, 8
    g = torch.Generator(device="cuda").manual_seed(7)
    q0, k0, v0 = (make(g, 1, h, P, 128) for h in (Hq, Hkv, Hkv))
    q, k, v = (make(g, B, h, T, 128) for h in (Hq, Hkv, Hkv))
    out0, out1 = torch.empty_like(q0), torch.empty_like(q)
    shape = pkg.shape_for_context(B, Hq, Hkv, 2, 32, T, 0.5, 2)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    layer = SharedPrefixLayer.from_prompts(shape, pkg.RotaryTable(), (q0, k0, v0), (q, k, v), out0, out1)
    assert torch.cuda.max_memory_allocated() - before < B * (k0.nbytes + v0.nbytes) // 2
    assert torch.equal(layer.k_prefix, k0)


@pytest.mark.parametrize("major", [False, True])
def test_prompt_outputs_in_either_layout(major):
    """Own tokens over prefix and own keys against 64 bits, written head-major or token-major, from views of one
    projection."""
    B, Hq, Hkv, P, T = 2, 8, 2, 333, 77
    g = torch.Generator(device="cuda").manual_seed(8)
    table = pkg.RotaryTable()
    q0, k0, v0 = (make(g, 1, h, P, 128) for h in (Hq, Hkv, Hkv))
    own = make(g, B, T, Hq + 2 * Hkv, 128)
    q, k, v = (own[:, :, a:b].transpose(1, 2) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv)))
    out0 = torch.empty_like(q0)
    out1 = torch.full((B, T, Hq, 128) if major else (B, Hq, T, 128), math.nan, dtype=torch.bfloat16, device="cuda")
    out1 = out1.transpose(1, 2) if major else out1
    shape = pkg.shape_for_context(B, Hq, Hkv, 2, 32, T, 0.3, 2)
    SharedPrefixLayer.from_prompts(shape, table, (q0, k0, v0), (q, k, v), out0, out1)
    mask = torch.arange(P + T, device="cuda") <= P + torch.arange(T, device="cuda")[:, None]
    for b in range(B):
        for h in range(Hq):
            keys, vals = torch.cat([k0[0, h // 4], k[b, h // 4]]), torch.cat([v0[0, h // 4], v[b, h // 4]])
            o, _, bound, _ = ref.attention(q[b, h], keys, vals, mask, SCALE)
            assert bool(((out1[b, h].double() - o).abs() <= bound).all())


@pytest.mark.parametrize("P", [0, 1, 129])
def test_short_prefixes_and_rows_of_any_alignment(P):
    """Prefixes of no and of one token; own rows that start and step at odd elements."""
    B, Hq, Hkv, T = 2, 4, 2, 33
    g = torch.Generator(device="cuda").manual_seed(11)
    table = pkg.RotaryTable()
    q0, k0, v0 = (make(g, 1, h, P, 128) for h in (Hq, Hkv, Hkv))
    q, k, v = (make(g, B, h, T, 131)[..., 1:129] for h in (Hq, Hkv, Hkv))
    out0, out1 = torch.empty_like(q0), torch.full((B, Hq, T, 128), math.nan, dtype=torch.bfloat16, device="cuda")
    layer = SharedPrefixLayer.from_prompts(pkg.shape_for_context(B, Hq, Hkv, 2, 32, T, 1.0, 2), table, (q0, k0, v0),
                                           (q, k, v), out0, out1)
    mask = torch.arange(P + T, device="cuda") <= P + torch.arange(T, device="cuda")[:, None]
    for b in range(B):
        for h in range(Hq):
            keys, vals = torch.cat([k0[0, h // 2], k[b, h // 2]]), torch.cat([v0[0, h // 2], v[b, h // 2]])
            o, _, bound, _ = ref.attention(q[b, h], keys, vals, mask, SCALE)
            assert bool(((out1[b, h].double() - o).abs() <= bound).all())
    out = torch.empty(B, Hq, 128, device="cuda")
    layer.step(*(make(g, B, h, 128) for h in (Hq, Hkv, Hkv)), out)
    layer.check()
    assert bool(torch.isfinite(out).all()) and layer.prefix == P


@pytest.mark.parametrize("call,at", [(None, 0), ("mikv_prompt_attention", 4), ("mikv_prefix_attention", 4),
                                     ("mikv_prefill_scores", 4)])
def test_check_reports_failures_of_the_prompts(monkeypatch, call, at):
    """A status word that one of the prompts' calls leaves (written by the host here) is still seen after the layer is
    built; without one nothing is reported."""
    from paper_2402_18096_gb300 import layer as module

    if call:
        real = getattr(module, call)

        def failing(*args, **kw):
            real(*args, **kw)
            args[at].view(torch.int32)[0] = 1

        monkeypatch.setattr(module, call, failing)
    layer = prompts(torch.Generator(device="cuda").manual_seed(9), 2, 4, 2, 60, 20, 0.5, 2)[0]
    monkeypatch.undo()
    out = torch.empty(2, 4, 128, dtype=torch.bfloat16, device="cuda")
    layer.step(*(torch.ones(2, h, 128, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2)), out)
    if call:
        with pytest.raises(pkg.MikvError) as e:
            layer.check()
        assert e.value.code == 6
    else:
        layer.check()


def test_refused_steps_change_nothing():
    """A full retained set and wrong arguments are refused before the new token is turned, inserted or counted."""
    B, Hq, Hkv = 2, 4, 2
    g = torch.Generator(device="cuda").manual_seed(10)
    layer = prompts(g, B, Hq, Hkv, 60, 20, 0.5, 2)[0]
    o, out = layer.own, torch.zeros(B, Hq, 128, dtype=torch.bfloat16, device="cuda")

    def refused(error, *args):
        c = o.cache
        state = [x for x in (c.k_hi, c.v_hi, c.hi_tok, c.acc, c.lo_tok, o.slots, *args)]
        before, counts = [x.clone() for x in state], (o.n_lo, o.pos)
        with pytest.raises(error) as e:
            layer.step(*args)
        assert all(torch.equal(x, y) for x, y in zip(state, before)) and counts == (o.n_lo, o.pos)
        return e.value

    q, k, v = (make(g, B, h, 128) for h in (Hq, Hkv, Hkv))
    refused(ValueError, q, k, v.float(), out)
    refused(ValueError, q, k, v[:1], out)
    refused(ValueError, q.float(), k, v, out)
    refused(ValueError, q, k.transpose(0, 1).contiguous().transpose(0, 1), v, out)
    refused(ValueError, q, k, v, out[:, :2])
    refused(ValueError, q, k, v, torch.zeros(B, Hq, 128, dtype=torch.float16, device="cuda"))
    while o.n_lo < o.shape.lo_cap:
        layer.step(*(make(g, B, h, 128) for h in (Hq, Hkv, Hkv)), out)
    assert refused(pkg.MikvError, q, k, v, out).code == 3


def snapshot(layer):
    """The own cache as the oracle's arrays."""
    c, s = layer.own.cache, layer.own.shape
    hi = {x: bits16(getattr(c, x)[:, :, :s.hi_cap].contiguous().cpu()) for x in ("k_hi", "v_hi")}
    hi.update({x: getattr(c, x)[:, :, :s.hi_cap].contiguous().cpu().numpy() for x in ("hi_tok", "acc")})
    lo = {x: getattr(c, x).cpu().numpy().copy() for x in ("k_codes", "v_codes", "lo_tok")}
    lo.update({x: getattr(c, x).cpu().numpy().view(np.uint16).copy() for x in ("k_params", "v_params")})
    return {**hi, **lo}, c.balancer.cpu().numpy()


@pytest.mark.parametrize("B,Hq,Hkv,P,T,bits", [(2, 8, 2, 700, 150, 2), (3, 4, 4, 130, 200, 4)])
def test_steps_over_prefix_and_retained_tokens(B, Hq, Hkv, P, T, bits):
    """Every step against the oracle on the cache as it stood before the step (its own insertion, attention over slots and
    retained rows, quantiser), joined in 64 bits with attention over the prefix."""
    steps = 4
    g = torch.Generator(device="cuda").manual_seed(6)
    layer, table, (k0, v0), (_, _, v_own) = prompts(g, B, Hq, Hkv, P, T, 0.2, steps, bits)
    o, G = layer.own, Hq // Hkv
    vmax = max(float(v0.abs().max()), float(v_own.abs().max()))
    full = torch.ones(G, P, dtype=torch.bool, device="cuda")
    for i in range(steps):
        q, k, v = (make(g, B, h, 128) for h in (Hq, Hkv, Hkv))
        tq, tk = q.clone(), k.clone()
        vmax = max(vmax, float(v.abs().max()))
        pkg.mikv_rotary(table, tq[:, :, None], tk[:, :, None], start=P + T + i)
        c, bal = snapshot(layer)
        n_lo, slots = o.n_lo, o.slots.cpu().numpy()
        out = torch.empty(B, Hq, 128, device="cuda")
        layer.step(q, k, v, out)
        oracle.insert_token(c, bits16(tk.cpu()), bits16(v.cpu()), T + i, slots)
        own, logits, ml = oracle.decode_attention(c, bits16(tq.cpu()), n_lo, SCALE, balancer_=bal)
        acc = torch.as_tensor(c["acc"]).double()
        rel = 0.0
        for b in range(B):
            for h in range(Hkv):
                hs = slice(h * G, (h + 1) * G)
                one = {x: c[x][b:b + 1, h:h + 1] for x in c}
                hi, lo = logit_bounds(one, bits16(tq[b:b + 1, hs].cpu()), bal[h], bits, 32, n_lo, SCALE)
                E, l_rtol = softmax_stat_bounds(hi, lo, o.shape.hi_cap + n_lo)
                mine = torch.as_tensor(E + l_rtol).cuda()
                po, pe, pb, peb = ref.attention(tq[b, hs], k0[0, h], v0[0, h], full, SCALE, out_dtype=torch.float32)
                jo, je, jb, jeb = ref.join(po, pe, pb, peb + mine, torch.as_tensor(own[b, hs]).cuda(),
                                           torch.as_tensor(ml[b, hs]).cuda(), torch.float32)
                # (the own part's documented bound is 2e-3 of the largest value)
                assert bool(((out[b, hs].double() - jo).abs() <= jb + 2e-3 * vmax).all())
                assert bool(((layer.ml[b, hs, 0].double() - je).abs() <= jeb).all())
                w = torch.exp(torch.as_tensor(logits[b, hs]) - je.cpu()[:, None]).sum(dim=0)
                acc[b, h] += w
                rel = max(rel, math.expm1(2 * float(jeb.max()) + 2 * float(hi.max())))
        got = o.cache.acc[:, :, :o.shape.hi_cap].cpu()
        assert bool(((got.double() - acc).abs() <= rel * acc + 2.0 ** -20 * acc).all())
        victim, _ = oracle.select_demote(got.numpy(), 1, ids=c["hi_tok"])
        assert np.array_equal(o.slots.cpu().numpy(), victim[:, :, 0])
        oracle.quantize_pack(c, c["k_hi"], c["v_hi"], victim, n_lo, src_tok=c["hi_tok"], balancer_=bal)
        after, _ = snapshot(layer)
        for x in ("k_codes", "v_codes", "k_params", "v_params", "lo_tok"):
            assert np.array_equal(after[x][:, :, :n_lo + 1], c[x][:, :, :n_lo + 1]), x
    assert o.n_lo == n_lo + 1 and o.pos == T + steps
