"""Prompts around the mixed-precision cache: rotary positions, prompt attention, attention over a shared prefix.

Like the rest of the binding, functions carry the C names (include/mikv.h holds their contracts) and only marshal
arguments. Tensors are taken as [batch, heads, tokens, 128] views with any strides the library allows: a projection's
token-major rows are passed as ``x.transpose(1, 2)``.
"""
from __future__ import annotations

import math
import struct

import torch

from . import HEAD_DIM, _check, _ptr, load

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
LAYOUTS = {"half": 0, "interleaved": 1}


# Descriptors and views are packed as bytes (ctypes passes their address): these calls are short enough that building
# ctypes structures would take longer than the launches.
_pack_view = struct.Struct("Pqqq").pack            # mikv_view
_pack_rotary = struct.Struct("9if").pack           # mikv_rotary_desc
_pack_prompt = struct.Struct("10iff").pack         # mikv_prompt_desc
_pack_prefix = struct.Struct("8iff").pack          # mikv_prefix_desc


def _dtype(t: torch.Tensor) -> int:
    code = DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"libmikv takes bfloat16, float16 or float32 tensors here, not {t.dtype}")
    return code


def _view(t: torch.Tensor, shape) -> bytes:
    """mikv_view of a [batch, heads, tokens, channels] tensor."""
    if t.shape != shape or len(shape) != 4:
        raise ValueError(f"expected a tensor of shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError("libmikv takes device tensors")
    b, h, n, c = t.stride()
    if c != 1:
        raise ValueError("the channels of a head must be contiguous")
    return _pack_view(t.data_ptr(), b, h, n)


def _dense(t, shape, dtype, name):
    """Pointer of an optional dense tensor after checking what the library cannot see."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr() if t.is_cuda and t.is_contiguous() else _ptr(t)


def _raw_stream(stream, t: torch.Tensor) -> int:
    """The given stream, or the current one of the tensor's device."""
    return torch._C._cuda_getCurrentRawStream(t.get_device()) if stream is None else stream.cuda_stream


def mikv_rotary_phases(frequencies) -> torch.Tensor:
    """int64 [n] (CPU): the bits of the phases (2^-64 turns per position) of angular frequencies in radians per
    position."""
    f = torch.as_tensor(frequencies, dtype=torch.float64).contiguous()
    out = torch.empty(f.numel(), dtype=torch.int64)
    _check("mikv_rotary_phases", load().mikv_rotary_phases(f.data_ptr(), f.numel(), out.data_ptr()))
    return out


def rotary_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       trained: int = 8192, slow: float = 1.0, fast: float = 4.0):
    """Angles per position of the rot_dim / 2 pairs, base^(-2 i / rot_dim), scaled for contexts `factor` times as long
    as was trained:
      "none"    as they are
      "linear"  all slowed by `factor`
      "base"    a raised base, base * factor^(rot_dim / (rot_dim - 2)): the slowest pair is slowed by `factor`, the
                fastest kept
      "bands"   by the turns a pair makes within `trained` positions: up to `slow` slowed by `factor`, from `fast` on
                kept, blended linearly between."""
    if scaling not in ("none", "linear", "base", "bands"):
        raise ValueError(f"rotary scaling {scaling!r}")
    if scaling == "base":
        if rot_dim <= 2:
            raise ValueError("a raised base needs at least two pairs")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = [base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]
    if scaling == "linear":
        return [x / factor for x in f]
    if scaling == "bands":
        blend = [min(1.0, max(0.0, (trained * x / (2 * math.pi) - slow) / (fast - slow))) for x in f]
        return [x * (w + (1.0 - w) / factor) for x, w in zip(f, blend)]
    return f


class RotaryTable:
    """What a model keeps for its rotary positions: the phases on the device, the pair layout, the number of turning
    channels and the factor on them. `frequencies` (radians per position) replaces base and scaling."""

    def __init__(self, head_dim: int = HEAD_DIM, rot_dim: int = None, base: float = 10000.0, layout: str = "half",
                 frequencies=None, amplitude: float = 1.0, device="cuda", **scaling):
        if layout not in LAYOUTS:
            raise ValueError(f"rotary layout {layout!r}: 'half' or 'interleaved'")
        self.head_dim = head_dim
        self.rot_dim = head_dim if rot_dim is None else rot_dim
        if self.rot_dim < 2 or self.rot_dim % 2 or self.rot_dim > head_dim:
            raise ValueError(f"rot_dim {self.rot_dim}: an even number of 2 .. {head_dim}")
        if frequencies is None:
            frequencies = rotary_frequencies(self.rot_dim, base, **scaling)
        if len(frequencies) != self.rot_dim // 2:
            raise ValueError(f"{self.rot_dim // 2} frequencies wanted, got {len(frequencies)}")
        self.layout = layout
        self.amplitude = float(amplitude)
        self.phases = mikv_rotary_phases(frequencies).to(device)


def mikv_rotary(table: RotaryTable, q, k=None, q_out=None, k_out=None, positions=None, start: int = 0,
                inverse: bool = False, stream=None):
    """Rotary positions of q [B, Hq, T, d] and, in the same launch, k [B, Hk, T, d]: into q_out / k_out, or in place
    where they are None. positions: int32 [B, T], or token t stands at start + t. inverse: the transposed map.
    Returns (q_out, k_out)."""
    q_out = q if q_out is None else q_out
    shape, dt = q.shape, q.dtype
    B, Hq, T, d = shape
    if q_out.dtype != dt:
        raise ValueError("rotary: inputs and outputs of one type")
    qi = _view(q, shape)
    qo = qi if q_out is q else _view(q_out, shape)
    Hk, ki, ko = 0, None, None
    if k is not None:
        k_out = k if k_out is None else k_out
        Hk = k.shape[1]
        shape = (B, Hk, T, d)
        if k.dtype != dt or k_out.dtype != dt:
            raise ValueError("rotary: inputs and outputs of one type")
        ki = _view(k, shape)
        ko = ki if k_out is k else _view(k_out, shape)
    desc = _pack_rotary(_dtype(q), B, T, Hq, Hk, d, table.rot_dim, LAYOUTS[table.layout], int(inverse), table.amplitude)
    rc = load().mikv_rotary(desc, qi, qo, ki, ko, _ptr(table.phases),
                            _dense(positions, (B, T), torch.int32, "positions"), start, _raw_stream(stream, q))
    _check("mikv_rotary", rc)
    return q_out, k_out


def mikv_mask_spans(spans, tk: int, q_start: int = None, causal: bool = True, docs=None, prefix=None, key_len=None,
                    stream=None):
    """The keys each query sees, into spans int32 [B, Tq, 2]. docs: int32 [B, n + 1] offsets of packed documents;
    prefix: int32 [B] (or [B, n] with docs); key_len: int32 [B]. q_start None: the queries are the last tokens."""
    B, tq, two = spans.shape
    if two != 2 or spans.dtype != torch.int32:
        raise ValueError("spans: int32 [B, Tq, 2]")
    n = 0 if docs is None else docs.shape[-1] - 1
    _check("mikv_mask_spans", load().mikv_mask_spans(
        _ptr(spans), B, tq, tk, tk - tq if q_start is None else q_start, int(causal),
        _dense(docs, (B, n + 1), torch.int32, "docs"), n,
        _dense(prefix, (B,) if docs is None or (prefix is not None and prefix.dim() == 1 and n == 1) else (B, n),
               torch.int32, "prefix"),
        _dense(key_len, (B,), torch.int32, "key_len"), _raw_stream(stream, spans)))


def _prompt_desc(q, k, out, causal, q_start, sm_scale, softcap) -> bytes:
    B, Hq, tq, d = q.shape
    Hkv, tk = k.shape[1:3]
    return _pack_prompt(_dtype(q), _dtype(out), B, Hq, Hkv, d, tq, tk, 1 if causal else 0,
                        tk - tq if q_start is None else q_start, 1.0 / math.sqrt(d) if sm_scale is None else sm_scale,
                        softcap)


def mikv_prompt_workspace_bytes(q, k) -> int:
    """Workspace of mikv_prompt_attention for q [B, Hq, Tq, d] and k [B, Hkv, Tk, d]."""
    return int(load().mikv_prompt_workspace_bytes(_prompt_desc(q, k, q, True, None, None, 0.0)))


def mikv_prompt_attention(q, k, v, out, workspace, sm_scale: float = None, causal: bool = True, q_start: int = None,
                          spans=None, softcap: float = 0.0, slopes=None, lse=None, stream=None):
    """Attention of a prompt: q [B, Hq, Tq, d] over k, v [B, Hkv, Tk, d] into out [B, Hq, Tq, d] (the inputs' type or
    float32). spans (mikv_mask_spans) or causal says which keys a query sees; softcap caps the scores, slopes
    float32 [Hq] add a distance bias; lse float32 [B, Hq, Tq] takes the log of each row's sum."""
    shape, ks = q.shape, k.shape
    B, Hq, tq, d = shape
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("prompt attention: q, k and v of one type")
    rc = load().mikv_prompt_attention(
        _prompt_desc(q, k, out, causal, q_start, sm_scale, softcap), _view(q, shape), _view(k, (B, ks[1], ks[2], d)),
        _view(v, ks), _view(out, shape), _dense(spans, (B, tq, 2), torch.int32, "spans"),
        _dense(slopes, (Hq,), torch.float32, "slopes"), _dense(lse, (B, Hq, tq), torch.float32, "lse"),
        _ptr(workspace), workspace.nbytes, _raw_stream(stream, q))
    _check("mikv_prompt_attention", rc)


def _prefix_desc(q, k, out, sm_scale, softcap) -> bytes:
    B, Hq, d = q.shape
    n, Hkv, P, _ = k.shape
    return _pack_prefix(_dtype(q), _dtype(out), B, n, Hq, Hkv, d, P,
                        1.0 / math.sqrt(d) if sm_scale is None else sm_scale, softcap)


def mikv_prefix_workspace_bytes(q, k) -> int:
    """Workspace of mikv_prefix_attention for q [B, Hq, d] and k [groups, Hkv, P, d]."""
    return int(load().mikv_prefix_workspace_bytes(_prefix_desc(q, k, q, None, 0.0)))


def mikv_prefix_attention(q, k, v, out, workspace, lens=None, q_pos=None, sm_scale: float = None,
                          softcap: float = 0.0, slopes=None, own_out=None, own_ml=None, ml=None, stream=None):
    """Single-token attention of q [B, Hq, d] over prefixes k, v [groups, Hkv, P, d] shared by B / groups requests
    each, into out [B, Hq, d]; lens int32 [groups] their lengths, q_pos int32 [B] the queries' positions. own_out
    float32 [B, Hq, d] and own_ml float32 [B, Hq, 2] (from mikv_decode_attention) join each request's own cache;
    ml float32 [B, Hq, 2] takes the joint (log-sum-exp, 1)."""
    shape, ks = q.shape, k.shape
    B, Hq, d = shape
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("prefix attention: q, k and v of one type")
    stat = (B, Hq, 2)
    rc = load().mikv_prefix_attention(
        _prefix_desc(q, k, out, sm_scale, softcap), _ptr(q), _view(k, (ks[0], ks[1], ks[2], d)), _view(v, ks),
        _dense(lens, ks[:1], torch.int32, "lens"), _dense(q_pos, (B,), torch.int32, "q_pos"),
        _dense(slopes, (Hq,), torch.float32, "slopes"), _dense(own_out, shape, torch.float32, "own_out"),
        _dense(own_ml, stat, torch.float32, "own_ml"), _dense(out, shape, out.dtype, "out"),
        _dense(ml, stat, torch.float32, "ml"), _ptr(workspace), workspace.nbytes, _raw_stream(stream, q))
    _check("mikv_prefix_attention", rc)
