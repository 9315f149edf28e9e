"""Host side of the entry points for drafted tokens (no GPU): refusals before anything is launched, workspace sizes, what the
binding checks, NVTX ranges."""
import ctypes
import math

import pytest
import torch

import paper_2402_18096_gb300 as pkg
import test_nvtx_ranges as ranges

P = 0x10000  # never dereferenced: validation rejects before any launch


@pytest.fixture(scope="module")
def lib():
    return pkg.load()


def shape(**kw):
    d = dict(batch=2, heads_q=8, heads_kv=2, head_dim=128, bits=2, group=32, hi_cap=17, hi_stride=32, lo_cap=64, hi_bits=16,
             hi_group=64, k_channel_group=0)
    d.update(kw)
    return pkg._Shape(*[d[n] for n, _ in pkg._Shape._fields_])


def cache(**kw):
    d = {n: P for n, _ in pkg._Cache._fields_}
    d.update(kw)
    return pkg._Cache(*[d[n] for n, _ in pkg._Cache._fields_])


def view(data=P, b=8 * 64 * 128, h=64 * 128, t=128):
    return pkg._View(data, b, h, t)


def lengths(n_hi=P, n_lo=P, slots=P, most=64):
    return pkg._Lengths(n_hi, n_lo, slots, most)


ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
NO = object()


def tree_rc(lib, s=None, c=None, masks=P, q=None, k=None, v=None, out=None, lens=None, lse=None, ws=P, n=1 << 40, **kw):
    d = dict(nodes=5, out_dtype=0, sm_scale=0.1)
    d.update(kw)
    desc = pkg._TreeDesc(*[d[x] for x, _ in pkg._TreeDesc._fields_])
    vs = [ref(x or view()) for x in (q, k, v, out)]
    return lib.mikv_tree_attention(ref(s or shape()), ref(c or cache()), ref(desc), masks, *vs,
                                   None if lens is NO else ref(lens or lengths()), lse, ws, n, None)


SHAPES = [(dict(head_dim=64), 2), (dict(heads_q=6), 2), (dict(heads_q=7), 1), (dict(batch=0), 1), (dict(bits=5), 2),
          (dict(group=16), 2), (dict(hi_bits=8), 2), (dict(k_channel_group=64, hi_stride=96), 2), (dict(hi_stride=24), 1),
          (dict(batch=40000), 2)]


@pytest.mark.parametrize("kw,code", SHAPES)
def test_shapes_refused(lib, kw, code):
    s = shape(**kw)
    assert tree_rc(lib, s) == code
    assert lib.mikv_tree_workspace_bytes(ref(s), 5) == 0 and lib.mikv_commit_workspace_bytes(ref(s), 5) == 0
    assert importance_rc(lib, s) == code
    assert commit_rc(lib, s) == code


def test_tree_arguments_refused(lib):
    assert lib.mikv_tree_workspace_bytes(ref(shape()), 5) >= 256
    assert lib.mikv_tree_workspace_bytes(ref(shape()), 0) == 0 == lib.mikv_tree_workspace_bytes(ref(shape()), 129)
    for name, t in (("k_hi", None), ("v_codes", None), ("k_params", P + 8), ("k_codes", P + 4), ("balancer", P + 4)):
        assert tree_rc(lib, c=cache(**{name: t})) == 1, name
    assert tree_rc(lib, masks=None) == 1 and tree_rc(lib, masks=P + 4) == 1
    assert tree_rc(lib, nodes=0) == 1 and tree_rc(lib, nodes=129) == 2
    assert tree_rc(lib, out_dtype=1) == 1 and tree_rc(lib, out_dtype=3) == 1
    for bad in (0.0, -1.0, math.inf, math.nan):
        assert tree_rc(lib, sm_scale=bad) == 1
    for name in ("q", "k", "v", "out"):
        assert tree_rc(lib, **{name: view(None)}) == 1
        assert tree_rc(lib, **{name: view(P + 8)}) == 1
        assert tree_rc(lib, **{name: view(t=132)}) == 1
        assert tree_rc(lib, **{name: view(t=0)}) == 1
        assert tree_rc(lib, **{name: view(b=0)}) == 1
        assert tree_rc(lib, **{name: view(h=-128)}) == 1
    assert tree_rc(lib, lens=lengths(most=65)) == 1 and tree_rc(lib, lens=lengths(most=-1)) == 1
    assert tree_rc(lib, lens=lengths(n_hi=P + 2)) == 1 and tree_rc(lib, lens=lengths(slots=P + 1)) == 1
    assert tree_rc(lib, s=shape(bits=0), lens=lengths(most=1)) == 1  # no retained set
    assert tree_rc(lib, lse=P + 2) == 1
    assert tree_rc(lib, ws=None) == 5 and tree_rc(lib, ws=P + 8) == 5 and tree_rc(lib, n=16) == 5
    assert lib.mikv_tree_attention(None, *[None] * 10, 0, None) == 1
    assert lib.mikv_tree_masks(None, None, P, 1, 1, None, 0, None) == 1
    assert lib.mikv_tree_masks(P, None, None, 1, 1, None, 0, None) == 1
    assert lib.mikv_tree_masks(P + 4, None, P, 1, 1, None, 0, None) == 1
    assert lib.mikv_tree_masks(P, None, P, 0, 1, None, 0, None) == 1
    assert lib.mikv_tree_masks(P, None, P, 1, 0, None, 0, None) == 1
    assert lib.mikv_tree_masks(P, None, P, 1, 129, None, 0, None) == 2


def importance_rc(lib, s=None, c=None, nodes=5, scale=0.1, path=P, steps=3, q=None, k=None, lse=P, lens=None, gained=P):
    return lib.mikv_path_importance(ref(s or shape()), ref(c or cache()), nodes, scale, path, steps, ref(q or view()),
                                    ref(k or view()), lse, ref(lens or lengths()), gained, None)


def commit_rc(lib, s=None, c=None, nodes=5, path=P, steps=3, k=None, v=None, gained=P, first=P, lens=None, out=None, next_=P,
              ws=P, n=256):
    return lib.mikv_commit_path(ref(s or shape()), ref(c or cache()), nodes, path, steps, ref(k or view()), ref(v or view()),
                                gained, first, None if lens is NO else ref(lens or lengths()), ref(out), next_, ws, n, None)


@pytest.mark.parametrize("kw", [dict(batch=30000, hi_cap=1 << 20, hi_stride=1 << 20), dict(batch=30000, lo_cap=2 ** 31 - 16)])
def test_trees_past_32_bits_refused(lib, kw):
    """Row numbers of the slots, and the costs that the work is divided by."""
    s = shape(**kw)
    assert lib.mikv_tree_workspace_bytes(ref(s), 5) == 0 and tree_rc(lib, s) == 2


def test_path_arguments_refused(lib):
    assert lib.mikv_commit_workspace_bytes(ref(shape()), 3) >= 256
    for rc in (importance_rc, commit_rc):
        assert rc(lib, path=None) == 1 and rc(lib, gained=None) == 1 and rc(lib, k=view(None)) == 1
        assert rc(lib, steps=0) == 1 and rc(lib, steps=129) == 2 and rc(lib, nodes=0) == 1 and rc(lib, nodes=200) == 2
        assert rc(lib, c=cache(acc=None)) == 1 and rc(lib, path=P + 2) == 1 and rc(lib, lens=lengths(most=65)) == 1
    assert importance_rc(lib, lse=None) == 1 and importance_rc(lib, scale=0.0) == 1 and importance_rc(lib, q=view(P + 2)) == 1
    assert commit_rc(lib, first=None) == 1 and commit_rc(lib, v=view(t=4)) == 1 and commit_rc(lib, lens=NO) == 1
    assert commit_rc(lib, out=lengths(n_lo=P + 2)) == 1 and commit_rc(lib, next_=P + 1) == 1
    assert commit_rc(lib, ws=None) == 5 and commit_rc(lib, n=255) == 5 and commit_rc(lib, ws=P + 16) == 5


def copy_rc(lib, pairs=((0, 1),), s=None, t=None, c=None, tc=None, lens=None, to=None, n=None):
    flat = [x for p in pairs for x in p]
    arr = (ctypes.c_int32 * max(len(flat), 1))(*flat)
    return lib.mikv_copy_requests(ref(s or shape()), ref(c or cache()), ref(t or shape()), ref(tc or cache()), arr,
                                  len(pairs) if n is None else n, ref(lens or lengths()), ref(to), None)


def test_copy_arguments_refused(lib):
    other = cache(k_hi=2 * P)
    assert copy_rc(lib, ()) == 0  # nothing to do: nothing is launched
    assert copy_rc(lib, ((0, 0),)) == 1                        # source and target in one cache
    assert copy_rc(lib, ((0, 2),)) == 1 and copy_rc(lib, ((2, 0),)) == 1 and copy_rc(lib, ((-1, 0),)) == 1
    assert copy_rc(lib, ((0, 1), (1, 0))) == 1
    assert copy_rc(lib, ((0, 1), (0, 1))) == 1                 # a target twice
    assert copy_rc(lib, ((0, 1), (1, 1)), tc=other) == 1
    assert copy_rc(lib, n=-1) == 1
    assert copy_rc(lib, c=cache(acc=P + 4)) == 1 and copy_rc(lib, tc=cache(lo_tok=P + 8)) == 1
    for kw in (dict(heads_q=8, heads_kv=4), dict(bits=3), dict(group=64), dict(hi_bits=8)):
        assert copy_rc(lib, t=shape(**kw), tc=other) == 1, kw
    assert copy_rc(lib, t=shape(hi_cap=16), tc=other) == 3
    assert copy_rc(lib, t=shape(lo_cap=48), tc=other) == 3
    assert copy_rc(lib, t=shape(lo_cap=80)) == 1               # one cache, two shapes
    assert copy_rc(lib, lens=lengths(most=80)) == 1
    assert copy_rc(lib, to=lengths(n_hi=P + 1)) == 1
    assert lib.mikv_copy_requests(None, None, None, None, None, 0, None, None, None) == 1


def test_copies_between_caches_that_share_some_arrays_refused(lib):
    for name in ("k_hi", "acc", "v_params", "lo_tok"):
        assert copy_rc(lib, ((0, 0),), tc=cache(**{name: 2 * P})) == 1, name
    assert copy_rc(lib, (), tc=cache(k_hi=2 * P)) == 1 and copy_rc(lib, (), tc=cache(**{n: 2 * P for n, _ in pkg._Cache._fields_})) == 0


def test_copies_that_read_lengths_they_write_refused(lib):
    """Two caches with one array of lengths: a row may keep its number, but not be read for one and written for another."""
    two = cache(**{n: 2 * P for n, _ in pkg._Cache._fields_})
    mine = dict(lens=lengths(n_hi=P, n_lo=2 * P, slots=3 * P), tc=two)
    for to in (lengths(n_hi=P, n_lo=None, slots=None), lengths(n_hi=None, n_lo=2 * P, slots=None),
               lengths(n_hi=None, n_lo=None, slots=3 * P)):
        assert copy_rc(lib, ((0, 1), (1, 0)), to=to, **mine) == 1
        assert copy_rc(lib, ((0, 0), (0, 1), (1, 2)), to=to, t=shape(batch=3), **mine) == 1


def test_copies_into_more_slots_than_are_counted_refused(lib):
    """All hi_cap slots in use, into a cache of more: only where the target's n_hi takes their number."""
    two = cache(**{n: 2 * P for n, _ in pkg._Cache._fields_})
    larger = dict(t=shape(hi_cap=18), tc=two)
    assert copy_rc(lib, (), lens=lengths(n_hi=None), **larger) == 3
    assert copy_rc(lib, (), lens=lengths(n_hi=None), to=lengths(n_hi=None), **larger) == 3
    none = lambda t, to: lib.mikv_copy_requests(ref(shape()), ref(cache()), ref(t), ref(two), (ctypes.c_int32 * 2)(), 0, None,  # noqa: E731
                                                ref(to), None)
    assert none(shape(hi_cap=18), None) == 3 and none(shape(), None) == 0
    assert copy_rc(lib, (), lens=lengths(n_hi=None), tc=two) == 0  # as many slots
    assert copy_rc(lib, (), lens=lengths(n_hi=None), to=lengths(n_hi=2 * P), **larger) == 0
    assert copy_rc(lib, (), **larger) == 0


def test_copies_of_free_slots_that_the_source_does_not_have_refused(lib):
    two = cache(**{n: 2 * P for n, _ in pkg._Cache._fields_})
    assert copy_rc(lib, (), lens=lengths(slots=None), to=lengths(), tc=two) == 1
    assert lib.mikv_copy_requests(ref(shape()), ref(cache()), ref(shape()), ref(two), (ctypes.c_int32 * 2)(), 0, None,
                                  ref(lengths()), None) == 1
    assert copy_rc(lib, (), lens=lengths(slots=None), to=lengths(slots=None), tc=two) == 0
    assert copy_rc(lib, (), lens=lengths(), to=lengths(slots=None), tc=two) == 0


def test_binding_refuses_what_the_library_cannot_see():
    s = pkg.Shape(1, 4, 2, 2, 32, 17, 32)
    arrays = [torch.zeros(1, 2, 32, 128, dtype=torch.bfloat16)] * 2 + \
        [torch.zeros(1, 2, 32, dtype=torch.int32), torch.zeros(1, 2, 32)] + \
        [torch.zeros(1, 2, 32, 32, dtype=torch.uint8)] * 2 + [torch.zeros(1, 2, 32, 4, 2, dtype=torch.float16)] * 2 + \
        [torch.zeros(1, 2, 32, dtype=torch.int32)]
    c = pkg.LayerCache.of(s, *arrays)
    for i in range(len(arrays)):
        with pytest.raises(ValueError):
            pkg.LayerCache.of(s, *[a[..., :-1] if j == i else a for j, a in enumerate(arrays)])
        with pytest.raises(ValueError):
            pkg.LayerCache.of(s, *[None if j == i else a for j, a in enumerate(arrays)])
    q = torch.zeros(1, 4, 3, 128, dtype=torch.bfloat16)
    k = torch.zeros(1, 2, 3, 128, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    masks = torch.zeros(1, 3, 4, dtype=torch.int32)
    with pytest.raises(ValueError):  # host tensors
        pkg.mikv_tree_attention(c, masks, q, k, k, q, ws)
    with pytest.raises(ValueError):
        pkg.mikv_tree_attention(c, masks, q.float(), k, k, q, ws)
    with pytest.raises(ValueError):
        pkg.mikv_tree_attention(c, masks, q, k, k, q.half(), ws)
    with pytest.raises(ValueError):
        pkg.mikv_copy_requests(c, c, [(0,)])


def test_ranges_of_the_new_entry_points(tmp_path, monkeypatch):
    monkeypatch.setattr(ranges, "CALLS", {
        "mikv_tree_masks": (None, None, None, 0, 0, None, 0, None),
        "mikv_tree_attention": (None,) * 11 + (0, None),
        "mikv_path_importance": (None, None, 0, 0.0, None, 0) + (None,) * 6,
        "mikv_commit_path": (None, None, 0, None, 0) + (None,) * 8 + (0, None),
        "mikv_copy_requests": (None,) * 5 + (0, None, None, None),
    })
    ranges.test_every_entry_point_has_one_balanced_range(tmp_path)
