"""Cases of the operators for drafted tokens over the mixed-precision cache: attention for a tree of drafted tokens,
the importance an accepted path hands out, its entry into the cache, and copies of whole requests.

Each case can be computed in its plain form (elementary torch operations in 32 bits) or through the framework's
entry points; `own` chooses. All sizes have head dimension 128, like the rest of the framework.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
OUTLIERS = (5, 69, 23, 87)  # key channels of large magnitude
BUFFERS = ("k_hi", "v_hi", "hi_tok", "acc", "k_codes", "v_codes", "k_params", "v_params", "lo_tok")


def tree_case(name, batch, hq, hkv, context, bits, group, ratio, nodes, tree, ragged):
    return {"name": name, "op": "tree", "batch": batch, "hq": hq, "hkv": hkv, "context": context, "bits": bits,
            "group": group, "ratio": ratio, "nodes": nodes, "tree": tree, "ragged": ragged}


def path_case(name, op, batch, hq, hkv, context, bits, group, ratio, nodes, steps, ragged):
    """op: "importance" or "commit" of up to `steps` accepted tokens out of `nodes` drafted ones."""
    return {"name": name, "op": op, "batch": batch, "hq": hq, "hkv": hkv, "context": context, "bits": bits,
            "group": group, "ratio": ratio, "nodes": nodes, "steps": steps, "ragged": ragged}


def copy_case(name, batch, copies, hkv, context, bits, group, ratio, ragged, same):
    """Each of `batch` requests copied to `copies` places; same: into free rows of its own cache, else into a cache
    with more retained rows."""
    return {"name": name, "op": "copy", "batch": batch, "copies": copies, "hkv": hkv, "context": context, "bits": bits,
            "group": group, "ratio": ratio, "ragged": ragged, "same": same}


def listed():
    return [
        # one request, a short context, a handful of drafted tokens: latency
        tree_case("tree-short", 1, 32, 32, 512, 4, 32, 0.2, 8, "random", False),
        # a full batch of long contexts, four query heads to a KV head
        tree_case("tree-long", 32, 32, 8, 32768, 2, 32, 0.2, 16, "binary", False),
        # requests of different lengths, one query head to a KV head, 3-bit codes, few tokens in a row
        tree_case("tree-ragged", 16, 40, 40, 8192, 3, 64, 0.1, 5, "chain", True),
        # a wide tree: every KV head has hundreds of query rows
        tree_case("tree-wide", 4, 32, 8, 16384, 4, 128, 0.25, 127, "random", False),
        # nothing in high precision but the drafted tokens
        tree_case("tree-codes-only", 8, 32, 32, 4096, 2, 32, 0.0, 33, "random", True),
        # the single token that a request without drafts decodes beside the others
        tree_case("tree-one-node", 33, 16, 8, 2047, 4, 64, 0.5, 1, "chain", True),
        # two accepted tokens of one request: latency
        path_case("importance-short", "importance", 1, 32, 32, 512, 4, 32, 0.2, 8, 2, False),
        # a full batch with paths of up to five tokens over a long context's important set
        path_case("importance-long", "importance", 32, 32, 8, 32768, 2, 32, 0.2, 16, 5, True),
        # two accepted tokens of one request enter its cache: latency
        path_case("commit-short", "commit", 1, 32, 32, 512, 4, 32, 0.2, 8, 2, False),
        # up to eight accepted tokens of 64 requests, 3-bit codes
        path_case("commit-batch", "commit", 64, 32, 32, 4096, 3, 128, 0.25, 16, 8, True),
        # one prompt's cache for four samples
        copy_case("copy-fork", 1, 3, 32, 512, 4, 32, 0.2, False, True),
        # requests of different lengths move, each twice, to a cache with room for more tokens
        copy_case("copy-grow", 8, 2, 40, 8192, 3, 64, 0.1, True, False),
    ]


def spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    hq, hkv = rng.choice(((32, 32), (40, 40), (32, 8), (16, 8), (8, 1), (4, 4)))
    kind = rng.choice(("tree", "tree", "tree", "importance", "commit", "copy"))
    context = spread(rng, 16, 32768)
    batch = spread(rng, 1, 64)
    while batch > 1 and batch * hkv * context > 32 * 8 * 32768 // (2 if kind == "copy" else 1):
        batch //= 2
    context = min(context, 32 * 8 * 32768 // (batch * hkv) // (2 if kind == "copy" else 1))
    bits, group, ratio = rng.choice((2, 3, 4)), rng.choice((32, 64, 128)), rng.choice((0.0, 0.05, 0.1, 0.2, 0.25, 0.5))
    ragged = rng.random() < 0.5
    if kind == "tree":
        nodes = spread(rng, 1, 128)
        while nodes > 1 and batch * hq * nodes * context > 32 * 32 * 16 * 32768:
            nodes = (nodes + 1) // 2 if nodes > 2 else 1
        c = tree_case("", batch, hq, hkv, context, bits, group, ratio, nodes,
                      rng.choice(("chain", "binary", "random")), ragged)
    elif kind == "copy":
        c = copy_case("", batch, spread(rng, 1, 3), hkv, context, bits, group, ratio, ragged, rng.random() < 0.5)
        while c["batch"] > 1 and c["batch"] * c["copies"] * hkv * context > 16 * 40 * 8192:
            c["batch"] //= 2
        while c["copies"] * c["batch"] * hkv * c["context"] > 16 * 40 * 8192:
            c["context"] = (c["context"] + 1) // 2
    else:
        nodes = spread(rng, 1, 64)
        c = path_case("", kind, batch, hq, hkv, context, bits, group, ratio, nodes, spread(rng, 1, min(nodes, 16)), ragged)
    del c["name"]
    return c


# ------------------------------------------------------------------ what a program has in hand

def budget(context, ratio):
    return int(math.floor(ratio * context + 0.5))


def lengths(case):
    """Important slots in use and retained rows of every request: a budget's share of its tokens, and the free slot."""
    n_hi, n_lo = [], []
    for b in range(case["batch"]):
        t = case["context"]
        if case["ragged"] and b > 0:
            t = 1 + random.Random(31 * b + t).randrange(t)
        k = min(budget(t, case["ratio"]), budget(case["context"], case["ratio"]))
        n_hi.append(k + 1)
        n_lo.append(t - k)
    return n_hi, n_lo


def caps(case):
    """Slots per head, rows allocated for them, retained rows allocated."""
    k = budget(case["context"], case["ratio"])
    return k + 1, (k + 16) // 16 * 16, (case["context"] - k + 64 + 15) // 16 * 16


def parents(case):
    """Parent of every drafted token (-1: the last token of the context itself); -2 behind a request's last one."""
    rows, n = [], case["nodes"]
    for b in range(case["batch"]):
        rng = random.Random(17 * b + n)
        tree = case.get("tree", "random")
        p = [i - 1 if tree == "chain" else (i - 1) // 2 if tree == "binary" and i else -1 if tree == "binary" else
             rng.randrange(max(-1, i - 6), i) for i in range(n)]
        used = rng.randrange(n + 1) if case["ragged"] and b % 4 == 3 else n
        rows.append([x if i < used else -2 for i, x in enumerate(p)])
    return rows


def ancestors(case):
    """bool [B, N, N] (CPU): node j is i or stands above it."""
    see = torch.zeros(case["batch"], case["nodes"], case["nodes"], dtype=torch.bool)
    for b, row in enumerate(parents(case)):
        for i, p in enumerate(row):
            if p >= -1:
                if p >= 0:
                    see[b, i] = see[b, p]
                see[b, i, i] = True
    return see


def paths(case):
    """Accepted nodes of every request, root first, -1 behind the last."""
    rows = []
    for b, row in enumerate(parents(case)):
        rng = random.Random(29 * b + case["steps"])
        used = [i for i, p in enumerate(row) if p >= -1]
        chain, i = [], max(rng.choice(used), rng.choice(used)) if used else -1
        while i >= 0:
            chain.insert(0, i)
            i = row[i]
        most = rng.randrange(case["steps"] + 1) if case["ragged"] else case["steps"]
        rows.append((chain[:most] + [-1] * case["steps"])[:case["steps"]])
    return rows


def normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def keys(gen, *shape):
    """Keys with the few channels of large magnitude that key caches show."""
    k = normal(gen, *shape)
    k[..., list(OUTLIERS)] *= 5
    return k


def fields(bits):
    """Of every channel: the 16-bit unit and the bit its code starts at (the two low bits and the high bit apart for 3
    bits, the high one's unit and bit after the first two)."""
    c = torch.arange(HEAD_DIM)
    u, m = c % 16, c // 16
    f = 2 if bits == 3 else bits
    per = 16 // f
    low = (8 * (2 * (m // per) + u // 8) + u % 8, f * (m % per))
    return low + ((16 + u % 8, 2 * m + u // 8) if bits == 3 else ())


def half_bits(x, up):
    """fp16 of x (fp32), rounded up or down."""
    h = x.to(torch.float16)
    wrong = h.float() < x if up else h.float() > x
    i = h.view(torch.int16).to(torch.int32)
    grow = (i >= 0) if up else (i < 0)  # away from zero in that direction: the next larger magnitude
    zero = (i & 0x7fff) == 0
    step = torch.where(zero, torch.where(torch.full_like(i, up, dtype=torch.bool), 1, -32767) - i,
                       torch.where(grow, 1, -1))
    return torch.where(wrong, i + step, i).to(torch.int16).view(torch.float16)


def quantize(x, bits, group):
    """Rows x [..., 128] (fp32) as packed codes [..., 16 bits] (uint8) and (scale, zero) pairs [..., 128 / group, 2]."""
    y = x.unflatten(-1, (-1, group))
    low, high = y.amin(-1), y.amax(-1)
    zero = half_bits(low, False)
    span = high - zero.float()
    most = torch.full_like(span, 2 ** bits - 1)
    scale = torch.where(span == 0, torch.ones_like(zero), half_bits(span / most, True))
    code = torch.round((y - zero.float()[..., None]) / scale.float()[..., None]).clamp(0, 2 ** bits - 1)
    code = code.flatten(-2).to(torch.int32)
    where = [w.to(x.device) for w in fields(bits)]
    units = torch.zeros(*x.shape[:-1], 8 * bits, dtype=torch.int32, device=x.device)
    units.index_add_(-1, where[0], (code & (3 if bits == 3 else 15)) << where[1].to(torch.int32))
    if bits == 3:
        units.index_add_(-1, where[2], (code >> 2) << where[3].to(torch.int32))
    return units.to(torch.int16).view(torch.uint8), torch.stack([scale, zero], dim=-1)


def make_cache(state, case, gen):
    """The arrays of a mixed-precision cache: random tokens split into important ones and coded ones."""
    b, h, bits, group = case["batch"], case["hkv"], case["bits"], case["group"]
    hi_cap, hi_stride, lo_cap = caps(case)
    n_hi, n_lo = lengths(case)
    most = max(n_lo)
    state["k_hi"], state["v_hi"] = keys(gen, b, h, hi_stride, HEAD_DIM), normal(gen, b, h, hi_stride, HEAD_DIM)
    k = keys(gen, b, h, most, HEAD_DIM)
    peak = torch.maximum(k.abs().amax((0, 2)) if most else k.new_zeros(h, HEAD_DIM), state["k_hi"].abs().amax((0, 2)))
    query = 3.0 + torch.rand(h, HEAD_DIM, generator=gen, device="cuda")  # largest magnitudes of a prompt's queries
    state["balancer"] = torch.sqrt(query / peak.float())
    state["k_codes"] = torch.zeros(b, h, lo_cap, 16 * bits, dtype=torch.uint8, device="cuda")
    state["v_codes"] = torch.zeros_like(state["k_codes"])
    state["k_params"] = torch.zeros(b, h, lo_cap, HEAD_DIM // group, 2, dtype=torch.float16, device="cuda")
    state["v_params"] = torch.zeros_like(state["k_params"])
    c, p = quantize(k.float() * state["balancer"][:, None], bits, group)
    state["k_codes"][:, :, :most], state["k_params"][:, :, :most] = c, p
    del k, c, p
    c, p = quantize(normal(gen, b, h, most, HEAD_DIM).float(), bits, group)
    state["v_codes"][:, :, :most], state["v_params"][:, :, :most] = c, p
    del c, p
    ids = torch.rand(b, h, hi_stride + lo_cap, generator=gen, device="cuda").argsort(dim=2).to(torch.int32)
    state["hi_tok"], state["lo_tok"] = ids[:, :, :hi_stride].contiguous(), ids[:, :, hi_stride:].contiguous()
    state["acc"] = torch.exp(torch.randn(b, h, hi_stride, generator=gen, device="cuda"))
    state["n_hi"] = torch.tensor(n_hi, dtype=torch.int32, device="cuda")
    state["n_lo"] = torch.tensor(n_lo, dtype=torch.int32, device="cuda")
    free = torch.rand(b, h, generator=gen, device="cuda") * state["n_hi"][:, None]
    state["slots"] = torch.minimum(free.to(torch.int32), state["n_hi"][:, None] - 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = dict(case)
    make_cache(state, case, gen)
    if case["op"] == "copy":
        prepare_copy(state, case)
    else:
        b, n = case["batch"], case["nodes"]
        # the rows that the projections of drafted tokens leave, token-major
        state["q"] = normal(gen, b, n, case["hq"], HEAD_DIM).transpose(1, 2)
        state["k"] = keys(gen, b, n, case["hkv"], HEAD_DIM).transpose(1, 2)
        state["v"] = normal(gen, b, n, case["hkv"], HEAD_DIM).transpose(1, 2)
        if case["op"] == "tree":
            prepare_tree(state, case)
        else:
            prepare_path(state, case, gen)
    if own:
        import paper_2402_18096_gb300 as pkg
        state["cache"] = wrap(pkg, state, "", case["hq"] if "hq" in case else case["hkv"])
        state["lens"] = pkg.Lengths(state["n_hi"], state["n_lo"], state["slots"])
        if case["op"] == "tree":
            state["masks"] = torch.empty(case["batch"], case["nodes"], 4, dtype=torch.int32, device="cuda")
            pkg.mikv_tree_masks(state["masks"], state["parents"])
            state["ws"] = torch.zeros(pkg.mikv_tree_workspace_bytes(state["cache"].shape, case["nodes"]),
                                      dtype=torch.uint8, device="cuda")
        elif case["op"] == "commit":
            state["lens_out"] = pkg.Lengths(state["n_hi_out"], state["n_lo_out"], state["slots"])
            state["ws"] = torch.zeros(pkg.mikv_commit_workspace_bytes(state["cache"].shape, case["steps"]),
                                      dtype=torch.uint8, device="cuda")
        elif case["op"] == "copy":
            state["to_cache"] = state["cache"] if case["same"] else wrap(pkg, state, "to_", case["hkv"])
            state["to_lens"] = pkg.Lengths(state["to_n_hi"], state["to_n_lo"], state["to_slots"])
    return state


def wrap(pkg, state, prefix, hq):
    """The framework's cache object around this state's arrays."""
    k_hi, codes = state[prefix + "k_hi"], state[prefix + "k_codes"]
    shape = pkg.Shape(k_hi.shape[0], hq, k_hi.shape[1], state["bits"], state["group"], caps(state)[0], codes.shape[2])
    return pkg.LayerCache.of(shape, *(state[prefix + x] for x in BUFFERS), balancer=state["balancer"])


def prepare_tree(state, case):
    state["parents"] = torch.tensor(parents(case), dtype=torch.int32, device="cuda")
    state["see"] = ancestors(case).cuda()
    b, n, hq = case["batch"], case["nodes"], case["hq"]
    state["out"] = torch.empty(b, n, hq, HEAD_DIM, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    state["lse"] = torch.empty(b, hq, n, dtype=torch.float32, device="cuda")


def prepare_path(state, case, gen):
    b, h, n, steps = case["batch"], case["hkv"], case["nodes"], case["steps"]
    state["path"] = torch.tensor(paths(case), dtype=torch.int32, device="cuda")
    # the sums that the tree's attention left: those over the important set, and what the others added
    s = state["q"].float().unflatten(1, (h, -1)).flatten(2, 3) @ state["k_hi"].float().transpose(2, 3)
    s = (s / math.sqrt(HEAD_DIM)).masked_fill(torch.arange(s.shape[3], device="cuda") >= state["n_hi"].view(-1, 1, 1, 1),
                                              -math.inf)
    state["lse"] = torch.logsumexp(s, dim=3).view(b, -1, n) + 0.5
    del s
    state["gained"] = torch.rand(b, h, steps, generator=gen, device="cuda") * 4
    state["first"] = state["n_hi"] - 1 + state["n_lo"]  # the position of a request's next token
    state["n_hi_out"], state["n_lo_out"] = torch.zeros_like(state["n_hi"]), torch.zeros_like(state["n_lo"])


def prepare_copy(state, case):
    b, copies = case["batch"], case["copies"]
    # each request's copies, in turn: (from, to)
    state["pairs"] = [[x, (b if case["same"] else 0) + x * copies + i] for x in range(b) for i in range(copies)]
    state["from_at"] = torch.tensor([p[0] for p in state["pairs"]], device="cuda")
    state["to_at"] = torch.tensor([p[1] for p in state["pairs"]], device="cuda")
    more = b * copies + (b if case["same"] else 0)
    lo_cap = state["k_codes"].shape[2] + (0 if case["same"] else 512)
    for x in BUFFERS:
        old = state[x]
        rows = old.shape[2] if x in ("k_hi", "v_hi", "hi_tok", "acc") else lo_cap
        new = torch.zeros(more, old.shape[1], rows, *old.shape[3:], dtype=old.dtype, device="cuda")
        if case["same"]:
            new[:b] = old
            state[x] = new
        state["to_" + x] = new
    for x in ("n_hi", "n_lo", "slots"):
        new = torch.zeros(more, *state[x].shape[1:], dtype=torch.int32, device="cuda")
        if case["same"]:
            new[:b] = state[x]
            state[x] = new
        state["to_" + x] = new


# ------------------------------------------------------------------ one pass

def run(state):
    if own:
        return run_own(state)
    return {"tree": plain_tree, "importance": plain_importance, "commit": plain_commit, "copy": plain_copy}[state["op"]](state)


def run_own(state):
    import paper_2402_18096_gb300 as pkg
    if state["op"] == "tree":
        pkg.mikv_tree_attention(state["cache"], state["masks"], state["q"], state["k"], state["v"], state["out"],
                                state["ws"], lens=state["lens"], lse=state["lse"])
        return {"out": state["out"], "lse": state["lse"]}
    if state["op"] == "importance":
        pkg.mikv_path_importance(state["cache"], state["path"], state["q"], state["k"], state["lse"], state["gained"],
                                 lens=state["lens"])
        return {"acc": state["acc"], "gained": state["gained"]}
    if state["op"] == "commit":
        pkg.mikv_commit_path(state["cache"], state["path"], state["k"], state["v"], state["gained"], state["first"],
                             state["ws"], lens=state["lens"], lens_out=state["lens_out"])
        return committed(state)
    pkg.mikv_copy_requests(state["cache"], state["to_cache"], state["pairs"], lens=state["lens"], to_lens=state["to_lens"])
    return copied(state)


def committed(state):
    return {x: state[x] for x in BUFFERS + ("n_hi_out", "n_lo_out")}


def copied(state):
    return {x: state["to_" + x] for x in BUFFERS + ("n_hi", "n_lo", "slots")}


def dequantize(codes, params, bits):
    """fp32 values of packed rows."""
    where = [w.to(codes.device) for w in fields(bits)]
    units = codes.view(torch.int16)
    code = (units[..., where[0]].to(torch.int32) >> where[1].to(torch.int32)) & (3 if bits == 3 else 2 ** bits - 1)
    if bits == 3:
        code += ((units[..., where[2]].to(torch.int32) >> where[3].to(torch.int32)) & 1) << 2
    code = code.to(torch.float32).unflatten(-1, (params.shape[-2], -1))
    return (code * params[..., :1].float() + params[..., 1:].float()).flatten(-2)


def important(state):
    """bool [B, Hkv, 1, slots]: the slots that hold a token."""
    i = torch.arange(state["k_hi"].shape[2], device=state["k_hi"].device)
    return ((i < state["n_hi"][:, None, None]) & (i != state["slots"][..., None]))[:, :, None]


def plain_tree(state):
    b, hq, n, d = state["q"].shape
    h, g, scale = state["hkv"], hq // state["hkv"], 1 / math.sqrt(HEAD_DIM)
    q = state["q"].float().reshape(b, h, g * n, d)
    k_lo = dequantize(state["k_codes"], state["k_params"], state["bits"])
    lo = (q / state["balancer"][:, None]) @ k_lo.transpose(2, 3) * scale
    del k_lo
    t = torch.arange(lo.shape[3], device=lo.device)
    lo = lo.masked_fill_(t >= state["n_lo"].view(-1, 1, 1, 1), -math.inf)
    hi = (q @ state["k_hi"].float().transpose(2, 3) * scale).masked_fill_(~important(state), -math.inf)
    see = state["see"][:, None, None].expand(b, 1, g, n, n).reshape(b, 1, g * n, n)
    own_part = (q @ state["k"].float().transpose(2, 3) * scale).masked_fill_(~see, -math.inf)
    real = see.any(dim=3, keepdim=True)
    m = torch.maximum(torch.maximum(lo.amax(3, keepdim=True), hi.amax(3, keepdim=True)), own_part.amax(3, keepdim=True))
    m = torch.where(m == -math.inf, 0.0, m)
    lo, hi, own_part = torch.exp(lo - m), torch.exp(hi - m), torch.exp(own_part - m)
    total = lo.sum(3, keepdim=True) + hi.sum(3, keepdim=True) + own_part.sum(3, keepdim=True)
    v_lo = dequantize(state["v_codes"], state["v_params"], state["bits"])
    out = lo @ v_lo + hi @ state["v_hi"].float() + own_part @ state["v"].float()
    out = torch.where(real, out / total, 0.0).view(b, hq, n, d).to(torch.bfloat16)
    lse = torch.where(real, m + torch.log(total), -math.inf).view(b, hq, n)
    return {"out": out, "lse": lse}


def accepted(state):
    """bool [B, steps], and the path with zeros behind the accepted nodes."""
    ok = (state["path"] >= 0).cumprod(dim=1).bool()
    return ok, torch.where(ok, state["path"], 0).to(torch.int64)


def rows_of(x, at):
    """x [B, H, N, ...] at the nodes `at` [B, P]."""
    return x.transpose(1, 2)[torch.arange(len(at), device=at.device)[:, None], at].transpose(1, 2)


def plain_importance(state):
    ok, at = accepted(state)
    b, p = at.shape
    h, g, scale = state["hkv"], state["hq"] // state["hkv"], 1 / math.sqrt(HEAD_DIM)
    q = rows_of(state["q"], at).float().reshape(b, h, g * p, HEAD_DIM)
    lse = rows_of(state["lse"], at).reshape(b, h, g * p, 1)
    live = ok[:, None, None].expand(b, 1, g, p).reshape(b, 1, g * p, 1)
    w = torch.exp(q @ state["k_hi"].float().transpose(2, 3) * scale - lse).masked_fill_(~(live & important(state)), 0.0)
    state["acc"] += w.sum(dim=2)
    k = rows_of(state["k"], at).float()
    w = torch.exp(q @ k.transpose(2, 3) * scale - lse)
    i = torch.arange(p, device=at.device)
    later = (i[:, None] >= i).repeat(g, 1)  # a node receives from itself and from those behind it
    w = w.masked_fill(~(live & ok[:, None, None] & later), 0.0)
    state["gained"].copy_(w.sum(dim=2))
    return {"acc": state["acc"], "gained": state["gained"]}


def order(score, ids):
    """One whole number per entry, ascending by score, then by id."""
    u = (score + 0.0).view(torch.int32).to(torch.int64)
    u = torch.where(u < 0, -1 - (u & 0x7fffffff), u)
    return u * 2 ** 32 + ids


def plain_commit(state):
    ok, at = accepted(state)
    b, p = at.shape
    h, cap, lo_cap = state["hkv"], caps(state)[0], state["k_codes"].shape[2]
    count = ok.sum(dim=1)
    held = state["n_hi"] - 1
    gone = (held + count - (cap - 1)).clamp(min=0)  # tokens that leave the important set
    fits = state["n_lo"] + gone <= lo_cap
    count, gone, ok = torch.where(fits, count, 0), torch.where(fits, gone, 0), ok & fits[:, None]
    step = torch.arange(p, device=at.device)
    new_tok = (state["first"][:, None] + step).expand(b, p)
    most = torch.iinfo(torch.int64).max
    old = order(state["acc"][:, :, :cap], state["hi_tok"][:, :, :cap]).masked_fill(~important(state)[:, :, 0, :cap], most)
    new = order(state["gained"], new_tok[:, None]).masked_fill(~ok[:, None], most)
    least = torch.sort(torch.cat([old, new], dim=2), dim=2, stable=True)[1][:, :, :p]  # in demotion order
    leaves = (step < gone[:, None])[:, None].expand(b, h, p)
    is_new = least >= cap
    slot, node = least.clamp(max=cap - 1), (least - cap).clamp(min=0)
    bi, hi = torch.arange(b, device=at.device)[:, None, None], torch.arange(h, device=at.device)[:, None]
    k_new, v_new = rows_of(state["k"], at), rows_of(state["v"], at)
    pick = is_new[..., None]
    k_out = torch.where(pick, k_new[bi, hi, node], state["k_hi"][bi, hi, slot]).float() * state["balancer"][:, None]
    v_out = torch.where(pick, v_new[bi, hi, node], state["v_hi"][bi, hi, slot]).float()
    tok_out = torch.where(is_new, new_tok[bi, node].to(torch.int32), state["hi_tok"][bi, hi, slot])
    row = (state["n_lo"][:, None, None] + step).expand(b, h, p)
    bx, hx, rx = bi.expand(b, h, p)[leaves], hi.expand(b, h, p)[leaves], row[leaves]
    for name, x in (("k", k_out), ("v", v_out)):
        codes, params = quantize(x[leaves], state["bits"], state["group"])
        state[name + "_codes"][bx, hx, rx], state[name + "_params"][bx, hx, rx] = codes, params
    state["lo_tok"][bx, hx, rx] = tok_out[leaves]
    # the tokens that stay take the slots of those that left, then slots not in use yet
    left = leaves & ~is_new
    rank = left.cumsum(dim=2) - 1
    freed = torch.zeros(b, h, p + 1, dtype=torch.int64, device=at.device)
    freed.scatter_(2, torch.where(left, rank, p), slot)
    demoted = torch.zeros(b, h, p + 1, dtype=torch.bool, device=at.device)
    demoted.scatter_(2, torch.where(leaves & is_new, node, p), True)
    stays = ok[:, None] & ~demoted[:, :, :p]
    place = stays.cumsum(dim=2) - 1
    many = left.sum(dim=2, keepdim=True)
    to = torch.where(place < many, freed.gather(2, place.clamp(min=0)), state["n_hi"][:, None, None] + place - many)
    bx, hx, to = bi.expand(b, h, p)[stays], hi.expand(b, h, p)[stays], to[stays]
    state["k_hi"][bx, hx, to], state["v_hi"][bx, hx, to] = k_new[stays], v_new[stays]
    state["hi_tok"][bx, hx, to] = new_tok[:, None].expand(b, h, p)[stays].to(torch.int32)
    state["acc"][bx, hx, to] = state["gained"][stays]
    state["n_hi_out"].copy_(state["n_hi"] + count - gone)
    state["n_lo_out"].copy_(state["n_lo"] + gone)
    return committed(state)


def plain_copy(state):
    src, dst = state["from_at"], state["to_at"]
    for x in BUFFERS:
        old, new = state[x], state["to_" + x]
        rows = min(old.shape[2], new.shape[2])
        n = state["n_hi"] if x in ("k_hi", "v_hi", "hi_tok", "acc") else state["n_lo"]
        live = torch.arange(rows, device=src.device) < n[src][:, None, None]
        live = live.view(*live.shape, *[1] * (old.dim() - 3))
        new[dst, :, :rows] = torch.where(live, old[src, :, :rows], new[dst, :, :rows])
    for x in ("n_hi", "n_lo", "slots"):
        state["to_" + x][dst] = state[x][src]
    return copied(state)


# ------------------------------------------------------------------ work and exact values

def row_bytes(case):
    """Bytes of a retained token's key and value."""
    return 2 * (16 * case["bits"] + 4 * HEAD_DIM // case["group"])


def work(case):
    n_hi, n_lo = (sum(x) for x in lengths(case))
    b, h = case["batch"], case["hkv"]
    if case["op"] == "copy":
        # read once, written once for each copy
        return {"bytes": h * (1 + case["copies"]) * (n_hi * 520 + n_lo * (row_bytes(case) + 4)), "flops": 0}
    hq, n = case["hq"], case["nodes"]
    if case["op"] == "tree":
        moved = h * (n_hi * 512 + n_lo * row_bytes(case)) + b * n * (h * 512 + hq * (512 + 4))
        return {"bytes": moved, "flops": 4 * HEAD_DIM * hq * n * (n_hi + n_lo) + 4 * HEAD_DIM * hq * int(ancestors(case).sum())}
    took = [sum(x >= 0 for x in p) for p in paths(case)]
    if case["op"] == "importance":
        live = sum(x for x, a in zip(lengths(case)[0], took) if a)
        return {"bytes": h * live * (256 + 8) + sum(took) * (hq * 260 + h * 260),
                "flops": 2 * HEAD_DIM * hq * sum(a * (x + a) for x, a in zip(lengths(case)[0], took))}
    moved = sum(8 * x for x, a in zip(lengths(case)[0], took) if a) + sum(took) * (512 * 3 + row_bytes(case) + 12)
    return {"bytes": h * moved, "flops": sum(took) * h * HEAD_DIM * 8}


def exact(case, seed):
    """The outputs in 64 bits, head by head from the definitions."""
    state = prepare(case, seed)
    if case["op"] == "tree":
        return exact_tree(case, state)
    if case["op"] == "importance":
        return exact_importance(case, state)
    return exact_commit(case, state) if case["op"] == "commit" else exact_copy(state)


def exact_codes(codes, params, case):
    """64-bit values of one head's rows, code by code from the layout of the planes."""
    word = codes.to(torch.int64)
    word = word[:, 0::2] + 256 * word[:, 1::2]
    x = torch.empty(len(codes), HEAD_DIM, dtype=torch.float64, device=codes.device)
    f = 2 if case["bits"] == 3 else case["bits"]
    for c in range(HEAD_DIM):
        m, u = divmod(c, 16)
        unit = 16 * (m // (16 // f)) + u
        code = torch.div(word[:, unit], 2 ** (f * (m % (16 // f))), rounding_mode="floor") % 2 ** f
        if case["bits"] == 3:
            code = code + 4 * (torch.div(word[:, 16 + u % 8], 2 ** (2 * m + u // 8), rounding_mode="floor") % 2)
        pair = params[:, c // case["group"]].double()
        x[:, c] = pair[:, 0] * code + pair[:, 1]
    return x


def exact_tree(case, state):
    b, hq, n, d = state["q"].shape
    g = hq // case["hkv"]
    out = torch.zeros(b, hq, n, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, hq, n), -math.inf, dtype=torch.float64, device="cuda")
    n_hi, n_lo = lengths(case)
    chains = parents(case)
    for x in range(b):
        for y in range(case["hkv"]):
            used = torch.arange(n_hi[x], device="cuda")
            used = used[used != state["slots"][x, y]]
            k_lo = exact_codes(state["k_codes"][x, y, :n_lo[x]], state["k_params"][x, y, :n_lo[x]], case)
            v_lo = exact_codes(state["v_codes"][x, y, :n_lo[x]], state["v_params"][x, y, :n_lo[x]], case)
            k = torch.cat([state["k_hi"][x, y, used].double(), k_lo / state["balancer"][y].double(), state["k"][x, y].double()])
            v = torch.cat([state["v_hi"][x, y, used].double(), v_lo, state["v"][x, y].double()])
            s = torch.einsum("gnd,td->gnt", state["q"][x, y * g:(y + 1) * g].double(), k) / math.sqrt(HEAD_DIM)
            hidden = torch.ones(n, n, dtype=torch.bool)
            for i in range(n):
                j = i if chains[x][i] >= -1 else -1
                while j >= 0:
                    hidden[i, j] = False
                    j = chains[x][j]
            s[:, :, -n:] = s[:, :, -n:].masked_fill(hidden.cuda(), -math.inf)
            real = torch.tensor([p >= -1 for p in chains[x]], device="cuda")
            e = torch.logsumexp(s, dim=2)
            lse[x, y * g:(y + 1) * g] = torch.where(real, e, -math.inf)
            out[x, y * g:(y + 1) * g] = torch.where(real[:, None], torch.exp(s - e[..., None]) @ v, 0.0)
    return {"out": out, "lse": lse}


def exact_importance(case, state):
    acc, gained = state["acc"].double(), torch.zeros_like(state["gained"], dtype=torch.float64)
    g, n_hi = case["hq"] // case["hkv"], lengths(case)[0]
    for x, path in enumerate(paths(case)):
        path = [i for i in path if i >= 0]
        for y in range(case["hkv"]):
            used = torch.arange(n_hi[x], device="cuda") != state["slots"][x, y]
            for at, i in enumerate(path):
                q = state["q"][x, y * g:(y + 1) * g, i].double()
                e = state["lse"][x, y * g:(y + 1) * g, i].double()[:, None]
                w = torch.exp(q @ state["k_hi"][x, y, :n_hi[x]].double().T / math.sqrt(HEAD_DIM) - e)
                acc[x, y, :n_hi[x]] += w.sum(dim=0) * used
                w = torch.exp(q @ state["k"][x, y, path[:at + 1]].double().T / math.sqrt(HEAD_DIM) - e)
                gained[x, y, :at + 1] += w.sum(dim=0)
    return {"acc": acc, "gained": gained}


def exact_commit(case, state):
    """The scores, and the pairs of the rows that were quantized: of each group the lowest value, and the step that
    reaches the highest one."""
    if case["batch"] * case["hkv"] * max(caps(case)[0], 150 * case["steps"]) > 3000000:
        return None
    n_hi, n_lo = lengths(case)
    acc, pairs = state["acc"].double(), {x: state[x].double() for x in ("k_params", "v_params")}
    cap = caps(case)[0]
    for x, path in enumerate(paths(case)):
        path = [i for i in path if i >= 0]
        gone = max(0, n_hi[x] - 1 + len(path) - (cap - 1))
        for y in range(case["hkv"]):
            score, tok = state["acc"][x, y].tolist(), state["hi_tok"][x, y].tolist()
            free = int(state["slots"][x, y])
            entries = [(score[s], tok[s], s, None) for s in range(n_hi[x]) if s != free]
            entries += [(float(state["gained"][x, y, i]), int(state["first"][x]) + i, None, i) for i in range(len(path))]
            leave = sorted(entries, key=lambda e: e[:2])[:gone]
            for j, (_, _, s, i) in enumerate(leave):
                for name, hi, new in (("k_params", "k_hi", "k"), ("v_params", "v_hi", "v")):
                    row = (state[hi][x, y, s] if i is None else state[new][x, y, path[i]]).double()
                    row = row * state["balancer"][y].double() if name == "k_params" else row
                    row = row.view(-1, case["group"])
                    low, high = row.amin(1), row.amax(1)
                    pairs[name][x, y, n_lo[x] + j, :, 0] = (high - low) / (2 ** case["bits"] - 1)
                    pairs[name][x, y, n_lo[x] + j, :, 1] = low
            places = [e[2] for e in leave if e[3] is None] + list(range(n_hi[x], cap))
            staying = [i for i in range(len(path)) if i not in [e[3] for e in leave]]
            for place, i in zip(places, staying):
                acc[x, y, place] = state["gained"][x, y, i].double()
    return {"acc": acc, **pairs}


def exact_copy(state):
    found = {x: state["to_" + x].double() for x in ("acc", "k_params", "v_params")}
    for a, b in state["pairs"]:
        hi, lo = int(state["n_hi"][a]), int(state["n_lo"][a])
        found["acc"][b, :, :hi] = state["acc"][a, :, :hi].double()
        for x in ("k_params", "v_params"):
            found[x][b, :, :lo] = state[x][a, :, :lo].double()
    return found
