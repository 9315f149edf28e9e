"""Cases of the attention-side operators: rotary positions, prompt attention with caps, biases and masks, and
single-token attention over a prefix that requests share.

Each case can be computed in its plain form (elementary torch operations in 32 bits) or through the framework's
entry points; `own` chooses. All sizes have head dimension 128, like the rest of the framework.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
OUTLIERS = ((5, 69), (23, 87))  # key channels of large magnitude and their rotary partners

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def rotary_case(name, batch, tokens, hq, hkv, dtype, layout, rot, scaling, inverse, token_major, per_request):
    return {"name": name, "op": "rotary", "batch": batch, "tokens": tokens, "hq": hq, "hkv": hkv, "dtype": dtype,
            "layout": layout, "rot": rot, "scaling": scaling, "inverse": inverse, "token_major": token_major,
            "per_request": per_request}


def prompt_case(name, batch, tq, tk, hq, hkv, dtype, cap, bias, docs, prefix, token_major):
    return {"name": name, "op": "prompt", "batch": batch, "tq": tq, "tk": tk, "hq": hq, "hkv": hkv, "dtype": dtype,
            "cap": cap, "bias": bias, "docs": docs, "prefix": prefix, "token_major": token_major}


def prefix_case(name, batch, groups, length, hq, hkv, dtype, cap, bias, ragged, joined):
    return {"name": name, "op": "prefix", "batch": batch, "groups": groups, "length": length, "hq": hq, "hkv": hkv,
            "dtype": dtype, "cap": cap, "bias": bias, "ragged": ragged, "joined": joined}


def listed():
    return [
        # one decoded token of 32 requests, each at its own position of a long context
        rotary_case("rotary-decode", 32, 1, 32, 8, "bf16", "half", 128, "none", False, False, True),
        # a whole long prompt as the projections leave it (token-major), turned into the cache's head-major rows,
        # frequencies scaled by wavelength for a longer context than was trained
        rotary_case("rotary-long-prompt", 1, 32768, 32, 8, "bf16", "half", 128, "bands", False, True, False),
        # the gradient's rotation: half of the head, adjacent pairs, 32-bit gradients, an odd length
        rotary_case("rotary-gradient", 3, 1021, 40, 40, "fp32", "interleaved", 64, "linear", True, False, False),
        # the shortest prompt: latency
        prompt_case("prompt-short", 1, 37, 37, 32, 32, "bf16", 0.0, False, 0, False, False),
        # causal prompts, four query heads to a KV head
        prompt_case("prompt-causal", 2, 8192, 8192, 32, 8, "bf16", 0.0, False, 0, False, False),
        # capped scores, each prompt with a prefix seen from both sides, odd length
        prompt_case("prompt-capped-prefix", 2, 2047, 2047, 32, 8, "fp16", 50.0, False, 0, True, False),
        # documents packed into rows with padding behind the last one, distance bias, token-major tensors
        prompt_case("prompt-packed-documents", 2, 4096, 4096, 40, 40, "bf16", 0.0, True, 9, False, True),
        # the next chunk of a few prompts over what is already in the cache
        prompt_case("prompt-chunk", 4, 64, 32768, 32, 8, "bf16", 0.0, False, 0, False, False),
        # one request, a short prompt, one query head to a KV head: latency
        prefix_case("prefix-one-request", 1, 1, 511, 32, 32, "bf16", 0.0, False, False, False),
        # 32 requests over one long prompt, joined with what each request's own cache gave
        prefix_case("prefix-shared-long", 32, 1, 32768, 32, 8, "bf16", 0.0, False, False, True),
        # four prompts of different lengths, four requests each; capped scores and distance bias
        prefix_case("prefix-four-prompts", 16, 4, 8192, 40, 40, "fp16", 30.0, True, True, True),
        # many requests over one prompt
        prefix_case("prefix-shared-wide", 256, 1, 8192, 32, 8, "bf16", 0.0, False, False, True),
    ]


def spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    hq, hkv = rng.choice(((32, 32), (40, 40), (32, 8), (16, 8), (8, 1), (4, 4)))
    kind = rng.choice(("rotary", "prompt", "prompt", "prefix", "prefix"))
    if kind == "rotary":
        tokens = spread(rng, 1, 32768)
        batch = spread(rng, 1, max(1, min(64, 32768 // tokens)))
        c = rotary_case("", batch, tokens, hq, hkv, rng.choice(("bf16", "fp16", "fp32")),
                        rng.choice(("half", "interleaved")), rng.choice((128, 128, 64, 32, 96)),
                        rng.choice(("none", "linear", "bands")), rng.random() < 0.4, rng.random() < 0.5,
                        rng.random() < 0.5)
        while c["batch"] * c["tokens"] * (hq + hkv) * (2 if c["dtype"] == "fp32" else 1) > 32768 * 40:
            c["tokens"] = (c["tokens"] + 1) // 2
    elif kind == "prompt":
        tk = spread(rng, 1, 32768)
        tq = tk if tk <= 8192 and rng.random() < 0.7 else spread(rng, 1, min(tk, 4096))
        batch = spread(rng, 1, 16)
        while batch > 1 and batch * hq * tq * tk > 2 * 32 * 8192 ** 2:
            batch //= 2
        while batch * hq * tq * tk > 2 * 32 * 8192 ** 2 // 2:
            tq = (tq + 1) // 2
        docs = rng.choice((0, 0, 1, 5, 17)) if tk >= 64 and tq == tk else 0
        c = prompt_case("", batch, tq, tk, hq, hkv, rng.choice(("bf16", "fp16")), rng.choice((0.0, 0.0, 30.0, 50.0)),
                        rng.random() < 0.35, docs, docs == 0 and tq == tk and rng.random() < 0.3, rng.random() < 0.5)
    else:
        length = spread(rng, 1, 32768)
        groups = rng.choice((1, 1, 1, 2, 5, 8))
        batch = groups * spread(rng, 1, 64)
        while batch > groups and batch * length > 256 * 8192:
            batch -= groups
        while groups * length * hkv > 32768 * 16:
            length = (length + 1) // 2
        c = prefix_case("", batch, groups, length, hq, hkv, rng.choice(("bf16", "fp16")),
                        rng.choice((0.0, 0.0, 30.0, 50.0)), rng.random() < 0.35, rng.random() < 0.5,
                        rng.random() < 0.6)
    del c["name"]
    return c


# ------------------------------------------------------------------ what a program has in hand

def normal(gen, *shape, dtype, token_major=False):
    """[B, H, T, d] standard normal; token_major: a view of a [B, T, H, d] tensor."""
    if token_major:
        b, h, t, d = shape
        return torch.randn(b, t, h, d, generator=gen, device="cuda", dtype=torch.float32).to(dtype).transpose(1, 2)
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def keys(gen, *shape, dtype, token_major=False):
    """Keys with the few channels of large magnitude that key caches show."""
    k = normal(gen, *shape, dtype=dtype, token_major=token_major)
    for a, b in OUTLIERS:
        k[..., a] *= 5
        k[..., b] *= 5
    return k


def slopes_of(heads):
    """Distance slopes 2^(-8 (h + 1) / heads) of the query heads."""
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def frequencies(rot, scaling):
    """Angles per position (radians) of the rot / 2 pairs, as Python floats."""
    f = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / 4.0 for x in f]
    if scaling == "bands":  # wavelengths over 8192 slowed by 8, under 2048 kept, blended between
        out = []
        for x in f:
            turns = 8192.0 * x / (2 * math.pi)
            blend = min(1.0, max(0.0, (turns - 1.0) / (4.0 - 1.0)))
            out.append(x * (blend + (1.0 - blend) / 8.0))
        return out
    return f


def documents(case):
    """Offsets [B][docs + 1] of the documents packed into each row (as many as fit, padding behind the last)."""
    rows = []
    for b in range(case["batch"]):
        rng = random.Random(1000 * b + case["tq"] + case["docs"])
        used = case["tq"] - case["tq"] // 32  # the tail is padding
        cuts = sorted(rng.randrange(used + 1) for _ in range(case["docs"] - 1))
        rows.append([0] + cuts + [used])
    return rows


def prefixes(case):
    """Length of the part of each prompt that all of its queries see."""
    return [random.Random(77 * b + case["tq"]).randrange(case["tq"] + 1) for b in range(case["batch"])]


def lengths(case):
    """Prefix length of each group of requests."""
    n, p = case["groups"], case["length"]
    if not case["ragged"]:
        return [p] * n
    return [p if g == 0 else random.Random(13 * g + p).randrange(p + 1) for g in range(n)]


def spans_of(case):
    """int64 [B, tq, 2]: the keys [lo, hi) that each query sees (CPU)."""
    b, tq, tk = case["batch"], case["tq"], case["tk"]
    pos = torch.arange(tq) + (tk - tq)
    lo = torch.zeros(b, tq, dtype=torch.int64)
    hi = (pos + 1).expand(b, tq).clone()
    if case["docs"]:
        off = torch.tensor(documents(case))
        last = off.shape[1] - 1
        at = torch.stack([torch.searchsorted(o, pos, right=True) - 1 for o in off])
        inside = at < last
        lo = torch.where(inside, torch.gather(off, 1, at.clamp(max=last - 1)), 0)
        hi = torch.where(inside, hi, 0)
    if case["prefix"]:
        hi = torch.maximum(hi, torch.tensor(prefixes(case))[:, None])
    return torch.stack([lo, hi], dim=2)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = dict(case)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "rotary":
        prepare_rotary(state, case, gen, dtype)
    elif case["op"] == "prompt":
        prepare_prompt(state, case, gen, dtype)
    else:
        prepare_prefix(state, case, gen, dtype)
    return state


def prepare_rotary(state, case, gen, dtype):
    b, t = case["batch"], case["tokens"]
    state["q"] = normal(gen, b, case["hq"], t, HEAD_DIM, dtype=dtype, token_major=case["token_major"])
    state["k"] = keys(gen, b, case["hkv"], t, HEAD_DIM, dtype=dtype, token_major=case["token_major"])
    first = torch.zeros(b, 1, dtype=torch.int64, device="cuda")
    if case["per_request"]:
        first = torch.randint(0, 32768, (b, 1), generator=gen, device="cuda")
    state["pos"] = (first + torch.arange(t, device="cuda")).to(torch.int32)
    f = frequencies(case["rot"], case["scaling"])
    # the turns per position as 64-bit fractions, so that position times frequency is exact modulo a turn
    turns = [round(x / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for x in f]
    state["phases"] = torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in turns], device="cuda")
    if own:
        import paper_2402_18096_gb300 as pkg
        state["table"] = pkg.RotaryTable(HEAD_DIM, rot_dim=case["rot"], frequencies=f, layout=case["layout"])
        state["q_out"] = torch.empty(b, case["hq"], t, HEAD_DIM, dtype=dtype, device="cuda")
        state["k_out"] = torch.empty(b, case["hkv"], t, HEAD_DIM, dtype=dtype, device="cuda")


def prepare_prompt(state, case, gen, dtype):
    b, tq, tk, major = case["batch"], case["tq"], case["tk"], case["token_major"]
    state["q"] = normal(gen, b, case["hq"], tq, HEAD_DIM, dtype=dtype, token_major=major)
    state["k"] = keys(gen, b, case["hkv"], tk, HEAD_DIM, dtype=dtype, token_major=major)
    state["v"] = normal(gen, b, case["hkv"], tk, HEAD_DIM, dtype=dtype, token_major=major)
    state["docs_at"] = torch.tensor(documents(case), dtype=torch.int32, device="cuda") if case["docs"] else None
    state["prefix_len"] = torch.tensor(prefixes(case), dtype=torch.int32, device="cuda") if case["prefix"] else None
    state["slopes"] = torch.tensor(slopes_of(case["hq"]), device="cuda") if case["bias"] else None
    if own:
        import paper_2402_18096_gb300 as pkg
        out = torch.empty(b, tq, case["hq"], HEAD_DIM, dtype=dtype, device="cuda").transpose(1, 2) if major else \
            torch.empty(b, case["hq"], tq, HEAD_DIM, dtype=dtype, device="cuda")
        state["out"] = out
        state["lse"] = torch.empty(b, case["hq"], tq, dtype=torch.float32, device="cuda")
        state["spans"] = torch.empty(b, tq, 2, dtype=torch.int32, device="cuda")
        state["ws"] = torch.zeros(pkg.mikv_prompt_workspace_bytes(state["q"], state["k"]), dtype=torch.uint8,
                                  device="cuda")


def prepare_prefix(state, case, gen, dtype):
    b, n, p, hq, hkv = case["batch"], case["groups"], case["length"], case["hq"], case["hkv"]
    state["q"] = normal(gen, b, hq, HEAD_DIM, dtype=dtype)
    state["k"] = keys(gen, n, hkv, p, HEAD_DIM, dtype=dtype)
    state["v"] = normal(gen, n, hkv, p, HEAD_DIM, dtype=dtype)
    state["lens"] = torch.tensor(lengths(case), dtype=torch.int32, device="cuda")
    mine = torch.randint(1, 65, (b,), generator=gen, device="cuda")  # own tokens of each request
    state["q_pos"] = (state["lens"].repeat_interleave(b // n) + mine).to(torch.int32)
    state["slopes"] = torch.tensor(slopes_of(hq), device="cuda") if case["bias"] else None
    state["own_out"] = state["own_ml"] = None
    if case["joined"]:  # what attention over each request's own tokens left: output, largest score, sum
        s = torch.randn(b, hq, 64, generator=gen, device="cuda") * 2
        s = s.masked_fill(torch.arange(64, device="cuda") >= mine[:, None, None], -math.inf)
        m = s.amax(dim=2)
        e = torch.exp(s - m[..., None])
        l = e.sum(dim=2)
        x = torch.randn(b, hq, 64, HEAD_DIM, generator=gen, device="cuda")
        state["own_out"] = ((e / l[..., None])[:, :, None] @ x)[:, :, 0].contiguous()
        state["own_ml"] = torch.stack([m, l], dim=2).contiguous()
    if own:
        import paper_2402_18096_gb300 as pkg
        state["out"] = torch.empty(b, hq, HEAD_DIM, dtype=dtype, device="cuda")
        state["ml"] = torch.empty(b, hq, 2, dtype=torch.float32, device="cuda")
        state["ws"] = torch.zeros(pkg.mikv_prefix_workspace_bytes(state["q"], state["k"]), dtype=torch.uint8,
                                  device="cuda")


# ------------------------------------------------------------------ one pass

def run(state):
    if own:
        return run_own(state)
    if state["op"] == "rotary":
        return plain_rotary(state)
    if state["op"] == "prompt":
        return plain_prompt(state)
    return plain_prefix(state)


def run_own(state):
    import paper_2402_18096_gb300 as pkg
    if state["op"] == "rotary":
        pkg.mikv_rotary(state["table"], state["q"], state["k"], state["q_out"], state["k_out"],
                        positions=state["pos"], inverse=state["inverse"])
        return {"q": state["q_out"], "k": state["k_out"]}
    if state["op"] == "prompt":
        spans = None
        if state["docs"] or state["prefix"]:
            spans = state["spans"]
            pkg.mikv_mask_spans(spans, state["tk"], causal=True, docs=state["docs_at"], prefix=state["prefix_len"])
        pkg.mikv_prompt_attention(state["q"], state["k"], state["v"], state["out"], state["ws"], causal=True,
                                  spans=spans, softcap=state["cap"], slopes=state["slopes"], lse=state["lse"])
        return {"out": state["out"], "lse": state["lse"]}
    pkg.mikv_prefix_attention(state["q"], state["k"], state["v"], state["out"], state["ws"], lens=state["lens"],
                              q_pos=state["q_pos"], softcap=state["cap"], slopes=state["slopes"],
                              own_out=state["own_out"], own_ml=state["own_ml"], ml=state["ml"])
    return {"out": state["out"], "ml": state["ml"]}


def plain_rotary(state):
    turn = (state["pos"].to(torch.int64)[..., None] * state["phases"]) >> 32  # modulo 2^64: a turn is 2^32 here
    angle = turn.to(torch.float32) * (2 * math.pi / 2.0 ** 32)
    if state["inverse"]:
        angle = -angle
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    return {"q": plain_turn(state, state["q"], c, s), "k": plain_turn(state, state["k"], c, s)}


def plain_turn(state, x, c, s):
    r = state["rot"]
    f = x.to(torch.float32)
    if state["layout"] == "half":
        a, b = f[..., :r // 2], f[..., r // 2:r]
        y = torch.cat([a * c - b * s, a * s + b * c, f[..., r:]], dim=-1)
    else:
        a, b = f[..., 0:r:2], f[..., 1:r:2]
        y = torch.cat([torch.stack([a * c - b * s, a * s + b * c], dim=-1).flatten(-2), f[..., r:]], dim=-1)
    return y.to(x.dtype).contiguous()


def visible(state, device):
    """bool [B, tq, tk]"""
    b, tq, tk = state["batch"], state["tq"], state["tk"]
    j = torch.arange(tk, device=device)
    i = torch.arange(tq, device=device) + (tk - tq)
    see = j <= i[:, None]
    if state["prefix"]:
        return see | (j < state["prefix_len"][:, None, None])
    if state["docs"]:
        at = state["docs_at"].to(torch.int64)
        doc = (j >= at[:, 1:, None]).sum(dim=1)  # documents that end at or before each token
        real = j < at[:, -1:]
        return see & (doc[:, :, None] == doc[:, None, :]) & real[:, :, None] & real[:, None, :]
    return see.expand(b, tq, tk)


def plain_softmax(s, v):
    """softmax(s) v and the log of the sum, for s [..., r, t] (masked entries -inf) and v [..., t, d]; rows with
    nothing visible give zeros."""
    m = s.amax(dim=-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    l = e.sum(dim=-1, keepdim=True)
    out = e @ v / torch.where(l == 0, 1.0, l)
    return out, (m + torch.log(l))[..., 0]


def plain_prompt(state):
    b, hq, tq, d = state["q"].shape
    hkv, tk = state["hkv"], state["tk"]
    q, k, v = (state[x].to(torch.float32) for x in "qkv")
    s = (q.reshape(b, hkv, -1, d) @ k.transpose(2, 3)).view(b, hkv, hq // hkv, tq, tk) * (1 / math.sqrt(d))
    if state["cap"]:
        s = state["cap"] * torch.tanh(s / state["cap"])
    if state["bias"]:
        i = torch.arange(tq, device=s.device) + (tk - tq)
        dist = (i[:, None] - torch.arange(tk, device=s.device)).abs()
        s = s - state["slopes"].view(hkv, -1, 1, 1) * dist
    s = s.masked_fill(~visible(state, s.device)[:, None, None], -math.inf)
    out, lse = plain_softmax(s.view(b, hkv, -1, tk), v)
    out = out.view(b, hq, tq, d).to(state["q"].dtype)
    return {"out": out, "lse": lse.view(b, hq, tq)}


def plain_prefix(state):
    b, hq, d = state["q"].shape
    n, hkv, p = state["groups"], state["hkv"], state["length"]
    per, g = b // n, hq // hkv
    q, k, v = (state[x].to(torch.float32) for x in "qkv")
    q = q.view(n, per, hkv, g, d).transpose(1, 2).reshape(n, hkv, per * g, d)
    s = (q @ k.transpose(2, 3)).view(n, hkv, per, g, p) * (1 / math.sqrt(d))
    if state["cap"]:
        s = state["cap"] * torch.tanh(s / state["cap"])
    j = torch.arange(p, device=s.device)
    if state["bias"]:
        dist = (state["q_pos"].view(n, 1, per, 1, 1) - j).abs()
        s = s - state["slopes"].view(1, hkv, 1, g, 1) * dist
    s = s.masked_fill(j >= state["lens"].view(n, 1, 1, 1, 1), -math.inf)
    out, lse = plain_softmax(s.view(n, hkv, per * g, p), v)
    out = out.view(n, hkv, per, g, d).transpose(1, 2).reshape(b, hq, d)
    lse = lse.view(n, hkv, per, g).transpose(1, 2).reshape(b, hq)
    if state["own_out"] is not None:
        mine = state["own_ml"][..., 0] + torch.log(state["own_ml"][..., 1])
        both = torch.logaddexp(lse, mine)
        out = out * torch.exp(lse - both)[..., None] + state["own_out"] * torch.exp(mine - both)[..., None]
        lse = both
    seen = lse != -math.inf
    return {"out": out.to(state["q"].dtype), "ml": torch.stack([lse, seen.to(torch.float32)], dim=2)}


# ------------------------------------------------------------------ work and exact values

def visible_pairs(case):
    s = spans_of(case)
    return int((s[..., 1] - s[..., 0]).clamp(min=0).sum())


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "rotary":
        x = case["batch"] * case["tokens"] * (case["hq"] + case["hkv"])
        return {"bytes": 2 * x * HEAD_DIM * size + 4 * case["batch"] * case["tokens"], "flops": 3 * x * case["rot"]}
    if case["op"] == "prompt":
        b, tq, tk, hq, hkv = (case[x] for x in ("batch", "tq", "tk", "hq", "hkv"))
        moved = b * (2 * tq * hq + 2 * tk * hkv) * HEAD_DIM * size + 4 * b * hq * tq
        return {"bytes": moved, "flops": 4 * HEAD_DIM * hq * visible_pairs(case)}
    b, n, hq, hkv = (case[x] for x in ("batch", "groups", "hq", "hkv"))
    total = sum(lengths(case))
    moved = 2 * total * hkv * HEAD_DIM * size + b * hq * (2 * HEAD_DIM * size + 8)
    moved += b * hq * (4 * HEAD_DIM + 8) if case["joined"] else 0
    return {"bytes": moved, "flops": 4 * HEAD_DIM * hq * (b // n) * total}


def exact(case, seed):
    """The outputs in 64 bits, head by head from the definitions."""
    state = prepare(case, seed)
    if case["op"] == "rotary":
        return exact_rotary(case, state)
    if case["op"] == "prompt":
        return exact_prompt(case, state)
    return exact_prefix(case, state)


def exact_rotary(case, state):
    f = torch.tensor(frequencies(case["rot"], case["scaling"]), dtype=torch.float64, device="cuda")
    a = state["pos"].double()[:, None, :, None] * f * (-1 if case["inverse"] else 1)
    z = torch.polar(torch.ones_like(a), a)
    found = {}
    for name in "qk":
        x = state[name].double()
        r = case["rot"]
        if case["layout"] == "half":
            pairs = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * z
            turned = torch.cat([pairs.real, pairs.imag], dim=-1)
        else:
            turned = torch.view_as_real(torch.view_as_complex(x[..., :r].unflatten(-1, (-1, 2)).contiguous()) * z)
            turned = turned.flatten(-2)
        found[name] = torch.cat([turned, x[..., r:]], dim=-1)
    return found


def exact_head(q, k, v, cap, slope, pos, spans):
    """out [r, d], lse [r] of query rows q [r, d] at positions pos over keys k, v [t, d], each row seeing
    keys [spans[:, 0], spans[:, 1])."""
    s = q.double() @ k.double().T / math.sqrt(HEAD_DIM)
    if cap:
        s = cap * torch.tanh(s / cap)
    j = torch.arange(k.shape[0], device=s.device)
    if slope is not None:
        s -= slope.double()[:, None] * (pos[:, None] - j).abs()
    s[(j < spans[:, :1]) | (j >= spans[:, 1:])] = -math.inf
    lse = torch.logsumexp(s, dim=1)
    w = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    return w @ v.double(), lse


def exact_prompt(case, state):
    b, hq, tq, d = state["q"].shape
    out = torch.empty(b, hq, tq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(b, hq, tq, dtype=torch.float64, device="cuda")
    spans = spans_of(case).cuda()
    pos = torch.arange(tq, device="cuda") + (case["tk"] - tq)
    for x in range(b):
        for h in range(hq):
            kv = h // (hq // case["hkv"])
            slope = state["slopes"][h].expand(tq) if case["bias"] else None
            out[x, h], lse[x, h] = exact_head(state["q"][x, h], state["k"][x, kv], state["v"][x, kv], case["cap"],
                                              slope, pos, spans[x])
    return {"out": out, "lse": lse}


def exact_prefix(case, state):
    b, hq, d = state["q"].shape
    per, g = b // case["groups"], hq // case["hkv"]
    out = torch.empty(b, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(b, hq, dtype=torch.float64, device="cuda")
    for x, length in enumerate(lengths(case)):
        rows = slice(x * per, (x + 1) * per)
        spans = torch.tensor([[0, length]], device="cuda").expand(per * g, 2)
        pos = state["q_pos"][rows].repeat_interleave(g)
        for kv in range(case["hkv"]):
            heads = slice(kv * g, (kv + 1) * g)
            slope = state["slopes"][heads].repeat(per) if case["bias"] else None
            o, e = exact_head(state["q"][rows, heads].reshape(-1, d), state["k"][x, kv], state["v"][x, kv],
                              case["cap"], slope, pos, spans)
            out[rows, heads], lse[rows, heads] = o.view(per, g, d), e.view(per, g)
    if case["joined"]:
        ml = state["own_ml"].double()
        weight = torch.stack([torch.exp(lse), torch.exp(ml[..., 0]) * ml[..., 1]], dim=-1)
        total = weight.sum(dim=-1)
        out = (out * weight[..., :1] + state["own_out"].double() * weight[..., 1:]) / total[..., None]
        lse = torch.log(total)
    return {"out": out, "ml": torch.stack([lse, (lse != -math.inf).double()], dim=2)}
