"""A batch of requests that share a long prompt prefix, through one layer: rotary positions, prompt attention, and
decode steps that join attention over the shared prefix (bf16, read once for the batch) with each request's own
mixed-precision cache. Random tensors stand in for a model's projections.

    python examples/shared_prompt.py [--requests 32 --prefix 8192 --own 512 --steps 8]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2402_18096_gb300 as pkg
from paper_2402_18096_gb300.layer import SharedPrefixLayer


def projections(gen, batch, heads_q, heads_kv, tokens, device):
    """q, k, v as views [B, H, T, d] of one token-major projection."""
    p = torch.randn(batch, tokens, heads_q + 2 * heads_kv, pkg.HEAD_DIM, generator=gen, device=device).to(torch.bfloat16)
    return tuple(p[:, :, a:b].transpose(1, 2) for a, b in
                 ((0, heads_q), (heads_q, heads_q + heads_kv), (heads_q + heads_kv, heads_q + 2 * heads_kv)))


def run(requests=32, prefix=8192, own=512, steps=8, heads_q=32, heads_kv=8, bits=2, group=32, ratio=0.2, device="cuda"):
    """Returns the decode outputs [steps, B, Hq, d] and the microseconds of a step."""
    gen = torch.Generator(device=device).manual_seed(0)
    d = pkg.HEAD_DIM
    table = pkg.RotaryTable(scaling="bands", factor=8.0, device=device)
    shape = pkg.shape_for_context(requests, heads_q, heads_kv, bits, group, own, ratio, steps)
    out0 = torch.empty(1, heads_q, prefix, d, dtype=torch.bfloat16, device=device)
    out1 = torch.empty(requests, heads_q, own, d, dtype=torch.bfloat16, device=device)
    layer = SharedPrefixLayer.from_prompts(shape, table, projections(gen, 1, heads_q, heads_kv, prefix, device),
                                           projections(gen, requests, heads_q, heads_kv, own, device), out0, out1)
    outs = torch.empty(steps, requests, heads_q, d, dtype=torch.bfloat16, device=device)
    new = [tuple(torch.randn(requests, h, d, generator=gen, device=device).to(torch.bfloat16)
                 for h in (heads_q, heads_kv, heads_kv)) for _ in range(steps)]
    first, last = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for i, (q, k, v) in enumerate(new):
        if i == min(3, steps - 1):
            first.record()
        layer.step(q, k, v, outs[i])
    last.record()
    torch.cuda.synchronize()
    layer.check()
    return outs, first.elapsed_time(last) * 1e3 / (steps - min(3, steps - 1))


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("requests", 32), ("prefix", 8192), ("own", 512), ("steps", 8)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args()
    outs, us = run(a.requests, a.prefix, a.own, a.steps)
    print(f"{a.requests} requests, shared prefix {a.prefix}, own tokens {a.own}: {us:.1f} us per decode step of one layer, "
          f"outputs finite: {bool(torch.isfinite(outs).all())}")


if __name__ == "__main__":
    main()
