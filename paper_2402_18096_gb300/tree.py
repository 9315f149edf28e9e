"""Drafted tokens over the mixed-precision cache: trees, their attention, the commit of an accepted path, copies of
requests.

Like the rest of the binding, functions carry the C names (include/mikv.h holds their contracts) and only marshal
arguments. Queries, keys and values of drafted tokens are [batch, heads, nodes, 128] views with any strides the library
allows: a projection's token-major rows are passed as ``x.transpose(1, 2)``.
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from . import HEAD_DIM, _check, _ptr, load
from .prompt import _dense, _raw_stream, _view

TREE_NODES = 128  # drafted tokens of a request at most

_OUT = {torch.bfloat16: 0, torch.float32: 2}
_I32, _F32, _BF16 = torch.int32, torch.float32, torch.bfloat16
_SCALE = 1.0 / math.sqrt(HEAD_DIM)
_pack_shape = struct.Struct("12i").pack     # mikv_shape
_pack_cache = struct.Struct("12P").pack     # mikv_cache
_pack_lengths = struct.Struct("PPPi").pack  # mikv_lengths
_pack_tree = struct.Struct("iif").pack      # mikv_tree_desc


class Lengths:
    """What the requests of a cache hold: n_hi int32 [B] slots in use, n_lo int32 [B] (or a number for all) retained rows,
    slots int32 [B, Hkv] the free slot among those in use. None: hi_cap slots, no rows, no slot free. n_lo_max bounds
    n_lo (None: the cache's lo_cap)."""

    def __init__(self, n_hi=None, n_lo=None, slots=None, n_lo_max: int = None):
        self.n_hi, self.slots = n_hi, slots
        self.n_lo = None if n_lo is None or isinstance(n_lo, int) else n_lo
        self.n_lo_max = n_lo if isinstance(n_lo, int) else 0 if n_lo is None else n_lo_max

    def _packed(self, shape) -> bytes:
        B, hi, lo, slots, most = (shape.batch,), self.n_hi, self.n_lo, self.slots, self.n_lo_max
        if most is None:
            most = shape.lo_cap if shape.bits else 0
        return _pack_lengths(0 if hi is None else _dense(hi, B, _I32, "n_hi"), 0 if lo is None else _dense(lo, B, _I32, "n_lo"),
                             0 if slots is None else _dense(slots, (shape.batch, shape.heads_kv), _I32, "slots"), most)


def _shape(s) -> bytes:
    return _pack_shape(s.batch, s.heads_q, s.heads_kv, s.head_dim, s.bits, s.group, s.hi_cap, s.hi_stride, s.lo_cap,
                       s.hi_bits, s.hi_group, s.k_channel_group)


def _cache(c) -> bytes:
    # (without a call for every array: 1 of the 10 us that a call takes on the host)
    return _pack_cache(*[0 if t is None else t.data_ptr() if t.is_cuda and t.is_contiguous() else _ptr(t)
                         for t in (c.k_hi, c.v_hi, c.hi_tok, c.acc, c.k_codes, c.v_codes, c.k_params, c.v_params,
                                   c.lo_tok, c.balancer, c.k_hi_params, c.v_hi_params)])


def _lens(lens, shape):
    return None if lens is None else lens._packed(shape)


def _bf16(names, *tensors):
    for t in tensors:
        if t.dtype != _BF16:
            raise ValueError(f"{', '.join(names)}: expected bfloat16, got {', '.join(str(x.dtype) for x in tensors)}")


def mikv_tree_masks(masks, parents, positions=None, first=None, start: int = 0, stream=None):
    """What the nodes of trees see of one another, into masks int32 [B, N, 4] (128 bits a node): parents int32 [B, N] holds
    the node before each one, -1 at a root, other numbers at padding. positions int32 [B, N] takes first int32 [B] (or
    `start`) plus a node's number of ancestors, for mikv_rotary."""
    B, N = parents.shape
    _check("mikv_tree_masks", load().mikv_tree_masks(
        _dense(masks, (B, N, 4), _I32, "masks"), _dense(positions, (B, N), _I32, "positions"),
        _dense(parents, (B, N), _I32, "parents"), B, N, _dense(first, (B,), _I32, "first"), start,
        _raw_stream(stream, parents)))


def mikv_tree_workspace_bytes(shape, nodes: int) -> int:
    return int(load().mikv_tree_workspace_bytes(_shape(shape), nodes))


def mikv_tree_attention(cache, masks, q, k, v, out, workspace, lens: Lengths = None, sm_scale: float = None, lse=None,
                        stream=None):
    """Attention of drafted tokens q [B, Hq, N, d] over the cache and, by masks (mikv_tree_masks), over their own k, v
    [B, Hkv, N, d], into out [B, Hq, N, d] (bfloat16 or float32); lse float32 [B, Hq, N] takes the log of each row's
    sum."""
    s = cache.shape
    N = q.shape[2]
    qs, ks = (s.batch, s.heads_q, N, HEAD_DIM), (s.batch, s.heads_kv, N, HEAD_DIM)
    _bf16("qkv", q, k, v)
    dt = _OUT.get(out.dtype)
    if dt is None:
        raise ValueError(f"out: expected bfloat16 or float32, got {out.dtype}")
    rc = load().mikv_tree_attention(
        _shape(s), _cache(cache), _pack_tree(N, dt, _SCALE if sm_scale is None else sm_scale),
        _dense(masks, (s.batch, N, 4), _I32, "masks"), _view(q, qs), _view(k, ks), _view(v, ks), _view(out, qs),
        _lens(lens, s), _dense(lse, qs[:3], _F32, "lse"), _ptr(workspace), workspace.nbytes,
        _raw_stream(stream, q))
    _check("mikv_tree_attention", rc)


def mikv_path_importance(cache, path, q, k, lse, gained, lens: Lengths = None, sm_scale: float = None, stream=None):
    """The importance that accepted paths (int32 [B, steps], nodes from the root on, any other number behind the last) hand
    out: added to cache.acc, and into gained float32 [B, Hkv, steps] for the paths' own nodes. q, k and lse are those of
    mikv_tree_attention."""
    s = cache.shape
    N, steps = q.shape[2], path.shape[-1]
    _bf16("qk", q, k)
    rc = load().mikv_path_importance(
        _shape(s), _cache(cache), N, _SCALE if sm_scale is None else sm_scale,
        _dense(path, (s.batch, steps), _I32, "path"), steps, _view(q, (s.batch, s.heads_q, N, HEAD_DIM)),
        _view(k, (s.batch, s.heads_kv, N, HEAD_DIM)), _dense(lse, (s.batch, s.heads_q, N), _F32, "lse"),
        _lens(lens, s), _dense(gained, (s.batch, s.heads_kv, steps), _F32, "gained"), _raw_stream(stream, q))
    _check("mikv_path_importance", rc)


def mikv_commit_workspace_bytes(shape, steps: int) -> int:
    return int(load().mikv_commit_workspace_bytes(_shape(shape), steps))


def mikv_commit_path(cache, path, k, v, gained, first, workspace, lens: Lengths, lens_out: Lengths = None, next=None,
                     stream=None):
    """Accepted paths enter the cache: their nodes (k, v [B, Hkv, N, d], tokens first[b] + step) join the important set
    with the scores `gained`, and what that then holds above its budget is demoted. lens_out (may be lens) takes the new
    n_hi and n_lo, next int32 [B] (may be first) the position behind the last token."""
    s = cache.shape
    N, steps = k.shape[2], path.shape[-1]
    ks = (s.batch, s.heads_kv, N, HEAD_DIM)
    _bf16("kv", k, v)
    rc = load().mikv_commit_path(
        _shape(s), _cache(cache), N, _dense(path, (s.batch, steps), _I32, "path"), steps, _view(k, ks),
        _view(v, ks), _dense(gained, (s.batch, s.heads_kv, steps), _F32, "gained"),
        _dense(first, (s.batch,), _I32, "first"), _lens(lens, s), _lens(lens_out, s),
        _dense(next, (s.batch,), _I32, "next"), _ptr(workspace), workspace.nbytes, _raw_stream(stream, k))
    _check("mikv_commit_path", rc)


def mikv_copy_requests(cache, to_cache, pairs, lens: Lengths = None, to_lens: Lengths = None, stream=None):
    """Whole requests copied: for every (from, to) of `pairs`, row `to` of to_cache takes what row `from` of cache holds
    (and to_lens its lengths). The two caches may be one, if no row is both source and target."""
    if any(len(p) != 2 for p in pairs):
        raise ValueError("pairs: (from, to) each")
    flat = [int(x) for p in pairs for x in p]
    rc = load().mikv_copy_requests(
        _shape(cache.shape), _cache(cache), _shape(to_cache.shape), _cache(to_cache),
        (ctypes.c_int32 * max(len(flat), 1))(*flat), len(pairs), _lens(lens, cache.shape),
        _lens(to_lens, to_cache.shape), _raw_stream(stream, cache.k_hi))
    _check("mikv_copy_requests", rc)
