"""Host side of the prompt, rotary and shared-prefix entry points (no GPU): refusals before anything is launched,
workspace sizes, phases of the rotary frequencies, NVTX ranges."""
import ctypes
import math

import pytest
import torch

import paper_2402_18096_gb300 as pkg
import test_nvtx_ranges as ranges
from paper_2402_18096_gb300.prompt import rotary_frequencies

P = 0x10000  # never dereferenced: validation rejects before any launch


@pytest.fixture(scope="module")
def lib():
    return pkg.load()


def view(data=P, b=8 * 64 * 128, h=64 * 128, t=128):
    return pkg._View(data, b, h, t)


def prompt_desc(**kw):
    d = dict(dtype=0, out_dtype=0, batch=2, heads_q=8, heads_kv=2, head_dim=128, tq=64, tk=64, causal=1, q_start=0,
             sm_scale=0.1, softcap=0.0)
    d.update(kw)
    return pkg._PromptDesc(*[d[n] for n, _ in pkg._PromptDesc._fields_])


def prompt_rc(lib, desc, q=None, k=None, v=None, out=None, spans=None, slopes=None, lse=None, ws=P, n=1 << 40):
    vs = [ctypes.byref(x or view()) for x in (q, k, v, out)]
    return lib.mikv_prompt_attention(ctypes.byref(desc), *vs, spans, slopes, lse, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=64), 2), (dict(heads_q=6), 2), (dict(heads_q=7), 1), (dict(heads_q=32), 2), (dict(batch=0), 1),
    (dict(tq=0), 1), (dict(tk=-1), 1), (dict(dtype=2), 1), (dict(dtype=3), 1), (dict(out_dtype=1), 1),
    (dict(sm_scale=0.0), 1), (dict(sm_scale=-1.0), 1), (dict(sm_scale=math.inf), 1), (dict(sm_scale=math.nan), 1),
    (dict(softcap=-1.0), 1), (dict(softcap=math.nan), 1), (dict(batch=70000), 2), (dict(q_start=1 << 30), 0),
    (dict(q_start=(1 << 30) + 1), 2), (dict(q_start=-(1 << 31)), 2)])
def test_prompt_shapes_refused(lib, kw, code):
    d = prompt_desc(**kw)
    if code == 0:  # accepted: checked through the pure workspace query instead of launching
        assert lib.mikv_prompt_workspace_bytes(ctypes.byref(d)) > 0
        return
    assert lib.mikv_prompt_workspace_bytes(ctypes.byref(d)) == 0
    assert prompt_rc(lib, d) == code


def test_prompt_arguments_refused(lib):
    d = prompt_desc()
    assert lib.mikv_prompt_workspace_bytes(ctypes.byref(d)) > 0
    assert prompt_rc(lib, d, q=view(None)) == 1
    for name in "qkv":
        assert prompt_rc(lib, d, **{name: view(P + 8)}) == 1      # alignment of the data
        assert prompt_rc(lib, d, **{name: view(t=132)}) == 1      # and of the strides
        assert prompt_rc(lib, d, **{name: view(t=-128)}) == 1
        assert prompt_rc(lib, d, **{name: view(t=0)}) == 1        # tokens are never shared
        assert prompt_rc(lib, d, **{name: view(b=1 << 40)}) == 1
    assert prompt_rc(lib, d, q=view(h=0)) == 1
    assert prompt_rc(lib, d, out=view(b=0)) == 1
    assert prompt_rc(lib, d, spans=P + 4) == 1
    assert prompt_rc(lib, d, ws=None) == 5
    assert prompt_rc(lib, d, ws=P + 8) == 5
    assert prompt_rc(lib, d, n=16) == 5
    assert lib.mikv_prompt_attention(None, *[None] * 7, None, 0, None) == 1


def prefix_rc(lib, q=P, k=None, v=None, own_out=None, own_ml=None, out=P, ws=P, n=1 << 40, **kw):
    d = dict(dtype=0, out_dtype=2, batch=8, groups=2, heads_q=8, heads_kv=2, head_dim=128, length=64, sm_scale=0.1,
             softcap=0.0)
    d.update(kw)
    desc = pkg._PrefixDesc(*[d[x] for x, _ in pkg._PrefixDesc._fields_])
    return lib.mikv_prefix_attention(ctypes.byref(desc), q, ctypes.byref(k or view()), ctypes.byref(v or view()), None,
                                     None, None, own_out, own_ml, out, None, ws, n, None)


def test_prefix_arguments_refused(lib):
    assert prefix_rc(lib, groups=3) == 1
    assert prefix_rc(lib, groups=0) == 1
    assert prefix_rc(lib, batch=0) == 1
    assert prefix_rc(lib, length=-1) == 1
    assert prefix_rc(lib, head_dim=256) == 2
    assert prefix_rc(lib, q=None) == 1
    assert prefix_rc(lib, q=P + 8) == 1
    assert prefix_rc(lib, out=P + 8) == 1
    assert prefix_rc(lib, own_out=P) == 1  # both parts of a join or none
    assert prefix_rc(lib, own_ml=P) == 1
    assert prefix_rc(lib, k=view(t=4)) == 1
    assert prefix_rc(lib, v=view(P + 2)) == 1
    assert prefix_rc(lib, n=8) == 5
    assert lib.mikv_prefix_attention(None, *[None] * 11, 0, None) == 1


def rotary_rc(lib, x=None, y=None, k=None, phases=P, **kw):
    d = dict(dtype=0, batch=2, tokens=4, heads_q=4, heads_k=0, head_dim=128, rot=128, layout=0, inverse=0,
             amplitude=1.0)
    d.update(kw)
    desc = pkg._RotaryDesc(*[d[n] for n, _ in pkg._RotaryDesc._fields_])
    k = ctypes.byref(k) if k else None
    return lib.mikv_rotary(ctypes.byref(desc), ctypes.byref(x or view()), ctypes.byref(y or view()), k, k, phases,
                           None, 0, None)


def test_rotary_arguments_refused(lib):
    assert rotary_rc(lib, phases=None) == 1
    assert rotary_rc(lib, x=view(None)) == 1
    assert rotary_rc(lib, x=view(P + 1)) == 1
    assert rotary_rc(lib, y=view(t=0)) == 1
    assert rotary_rc(lib, heads_k=2) == 1  # no second tensor given
    assert rotary_rc(lib, rot=0) == 1
    assert rotary_rc(lib, rot=3) == 1
    assert rotary_rc(lib, rot=130) == 1
    assert rotary_rc(lib, layout=2) == 1
    assert rotary_rc(lib, dtype=5) == 1
    assert rotary_rc(lib, head_dim=64, rot=64) == 2
    assert rotary_rc(lib, amplitude=math.nan) == 1
    assert rotary_rc(lib, tokens=0) == 0  # nothing to do: nothing is launched
    assert lib.mikv_mask_spans(None, 1, 1, 1, 0, 1, None, 0, None, None, None) == 1
    assert lib.mikv_mask_spans(P + 4, 1, 1, 1, 0, 1, None, 0, None, None, None) == 1
    assert lib.mikv_mask_spans(P, 1, 1, 1, 0, 1, P, 0, None, None, None) == 1
    assert lib.mikv_mask_spans(P, 1, 0, 1, 0, 1, None, 0, None, None, None) == 0


def test_workspace_grows_with_the_problem(lib):
    sizes = [lib.mikv_prompt_workspace_bytes(ctypes.byref(prompt_desc(tk=n))) for n in (0, 1, 64, 1000, 30000)]
    assert all(s >= 256 for s in sizes) and sizes == sorted(sizes)


def test_phases():
    """Phases are the turns per position as 64-bit fractions, to the last bits that doubles hold."""
    f = rotary_frequencies(128) + [0.0, 2 * math.pi, 100.0]
    got = pkg.mikv_rotary_phases(f).tolist()
    for x, p in zip(f, got):
        want = (x / (2 * math.pi)) % 1.0
        d = abs((p % 2 ** 64) / 2 ** 64 - want)
        assert min(d, 1 - d) <= 2.0 ** -52
    assert got[-3] == 0
    for bad in (-1.0, math.nan, math.inf):
        with pytest.raises(pkg.MikvError):
            pkg.mikv_rotary_phases([bad])


def test_binding_refuses_what_the_library_cannot_see():
    q = torch.zeros(1, 4, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # host tensors
        pkg.mikv_prompt_attention(q, q, q, q, torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(ValueError):
        pkg.mikv_rotary(pkg.RotaryTable(device="cpu"), q)
    with pytest.raises(ValueError):
        rotary_frequencies(128, scaling="cubic")
    with pytest.raises(ValueError):
        pkg.RotaryTable(frequencies=[1.0], device="cpu")


def test_ranges_of_the_new_entry_points(tmp_path, monkeypatch):
    monkeypatch.setattr(ranges, "CALLS", {
        "mikv_rotary": (None, None, None, None, None, None, None, 0, None),
        "mikv_mask_spans": (None, 0, 0, 0, 0, 0, None, 0, None, None, None),
        "mikv_prompt_attention": (None,) * 9 + (0, None),
        "mikv_prefix_attention": (None,) * 12 + (0, None),
    })
    ranges.test_every_entry_point_has_one_balanced_range(tmp_path)
