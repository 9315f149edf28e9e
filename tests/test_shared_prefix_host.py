"""Host side of the shared-prefix layer and of the rotary binding (no GPU): what they refuse before anything is
launched."""
import ctypes

import pytest
import torch

import paper_2402_18096_gb300 as pkg
import test_nvtx_ranges as ranges
from paper_2402_18096_gb300 import prompt
from paper_2402_18096_gb300.layer import SharedPrefixLayer


def test_key_lengths_are_refused():
    """Requests of several lengths: the own caches hold the same number of tokens for every request, so padding would be
    kept and attended. Refused before anything is turned."""
    B, Hq, Hkv, P, T = 2, 4, 2, 8, 6
    shape = pkg.shape_for_context(B, Hq, Hkv, 2, 32, T, 0.5, 1)
    prefix = tuple(torch.ones(1, h, P, 128, dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    own = tuple(torch.ones(B, h, T, 128, dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    with pytest.raises(ValueError, match="key_len"):
        SharedPrefixLayer.from_prompts(shape, pkg.RotaryTable(device="cpu"), prefix, own, torch.empty_like(prefix[0]),
                                       torch.empty_like(own[0]),
                                       key_len=torch.tensor([P + T, P + 2], dtype=torch.int32))
    assert all(bool((x == 1).all()) for x in prefix + own)


def test_no_tokens_need_no_arrays():
    """Empty tensors have no address: with no tokens nothing is launched and no pointer is asked for."""
    lib = pkg.load()
    view = pkg._View(None, 0, 0, 0)
    args = [ctypes.byref(view)] * 4

    def rotary(tokens, **kw):
        d = dict(dtype=0, batch=2, tokens=tokens, heads_q=4, heads_k=2, head_dim=128, rot=128, layout=0, inverse=0,
                 amplitude=1.0)
        d.update(kw)
        return lib.mikv_rotary(ctypes.byref(pkg._RotaryDesc(*[d[n] for n, _ in pkg._RotaryDesc._fields_])), *args,
                               0x10000, None, 0, None)

    assert rotary(0) == 0
    assert rotary(1) == 1 and rotary(-1) == 1
    assert rotary(0, rot=3) == 1 and rotary(0, dtype=7) == 1 and rotary(0, head_dim=64, rot=64) == 2
    assert lib.mikv_mask_spans(None, 2, 0, 5, 0, 1, None, 0, None, None, None) == 0
    assert lib.mikv_mask_spans(None, 2, 1, 5, 0, 1, None, 0, None, None, None) == 1
    assert lib.mikv_mask_spans(None, 0, 0, 5, 0, 1, None, 0, None, None, None) == 1


def test_given_normalisers_refused():
    """mikv_prefill_scores_lse: what is checked before anything is launched."""
    lib, p = pkg.load(), 0x10000  # never dereferenced
    shape = pkg.Shape(2, 8, 2, 2, 32, 1, 16)

    def rc(q=p, k=p, T=64, lse=p, scores=p, ws=p, n=1 << 30, s=shape):
        return lib.mikv_prefill_scores_lse(s.c(), q, k, T, 0.1, lse, scores, ws, n, None)

    assert rc(lse=None) == 1 and rc(lse=p + 2) == 1
    assert rc(q=None) == 1 and rc(k=p + 8) == 1 and rc(scores=None) == 1 and rc(T=0) == 1
    assert rc(s=pkg.Shape(2, 7, 2, 2, 32, 1, 16)) != 0
    assert rc(ws=None) == 5 and rc(n=16) == 5
    q = torch.zeros(2, 8, 64, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="lse"):
        pkg.mikv_prefill_scores(shape, q, q[:, :2], torch.zeros(2, 2, 64), q, lse=torch.zeros(2, 8, 63))


def test_range_of_the_given_form(tmp_path, monkeypatch):
    monkeypatch.setattr(ranges, "CALLS", {"mikv_prefill_scores_lse": (None, None, None, 0, 1.0, None, None, None, 0, None)})
    ranges.test_every_entry_point_has_one_balanced_range(tmp_path)


def test_phases_on_the_host_are_refused(monkeypatch):
    """The kernel reads the phases: a table on the host must not reach it (as with every other pointer)."""
    calls = []

    class Library:
        def mikv_rotary(self, *args):
            calls.append(args)
            return 0

    monkeypatch.setattr(prompt, "load", Library)
    monkeypatch.setattr(prompt, "_view", lambda t, shape: b"")
    monkeypatch.setattr(prompt, "_raw_stream", lambda stream, t: 0)
    table = pkg.RotaryTable.__new__(pkg.RotaryTable)
    table.rot_dim, table.layout, table.amplitude = 128, "half", 1.0
    table.phases = torch.zeros(64, dtype=torch.int64)
    with pytest.raises(ValueError, match="device"):
        prompt.mikv_rotary(table, torch.zeros(1, 1, 1, 128))
    assert not calls
