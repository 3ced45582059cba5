"""A routed feed-forward layer served from packed experts.

Every expert's matrices are coded by the codec, as they would be stored; to serve them they are decoded to bf16 and, for the 8-bit
layer, quantised once more to 8-bit integers with a scale for each output channel.  A pass is: logits to experts, tokens to 8
bits, the gate and up projections of the chosen experts with silu(gate) * up, that to 8 bits, the down projections, and the weighted
sum back to the tokens.

    python examples/routed_layer.py [--tokens 256] [--experts 16] [--choices 2] [--width 2048] [--hidden 1024]
"""
from __future__ import annotations

import argparse
import collections
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_26339_amd import qamw, synth  # noqa: E402

Experts = collections.namedtuple("Experts", "weights scales")      # [n][outputs][inputs]; [n][outputs] for 8 bits, None for bf16


def stored_and_decoded(matrices, bits=11, block=128):
    """What a loader finds in a checkpoint and makes of it: n matrices [outputs][inputs] through the codec, decoded to bf16."""
    codebook = torch.from_numpy(qamw.train_codebook(bits, 1 << 16, max_iters=40)[0]).to(matrices.device)
    out = torch.empty(matrices.shape, dtype=torch.bfloat16, device=matrices.device)
    for W, to in zip(matrices, out):
        sigma = qamw.calibrate_sigma(W, block)
        packed, norms = qamw.encode(W, codebook, bits, block, pair_sigma=sigma)
        qamw.decode(packed, norms, W.shape[1], codebook, bits, block, pair_sigma=sigma, out=to)
    return Experts(out, None)


def in_8_bits(experts):
    """The same experts with every output channel in 8-bit integers."""
    n, outs, ins = experts.weights.shape
    codes, scales = qamw.int8_quantize(experts.weights.view(n * outs, ins))
    return Experts(codes.view(n, outs, ins), scales.view(n, outs))


def routed_layer(x, logits, up, down, choices):
    """x [tokens][width] bf16, logits [tokens][experts]; up [n][2 hidden][width] (gates, then up projections), down [n][width][hidden],
    both in 8 bits or both in bf16.  Returns [tokens][width] bf16."""
    r = qamw.route(logits, choices)
    if up.scales is None:
        h = qamw.grouped_matmul(x, up.weights, r.offsets, rows=r.rows, gated=True)
        y = qamw.grouped_matmul(h, down.weights, r.offsets)
    else:
        codes, scales = qamw.int8_quantize(x)                       # once a token, however many experts it has
        h = qamw.grouped_matmul(codes, up.weights, r.offsets, rows=r.rows, x_scales=scales, w_scales=up.scales, gated=True)
        codes, scales = qamw.int8_quantize(h)
        y = qamw.grouped_matmul(codes, down.weights, r.offsets, x_scales=scales, w_scales=down.scales)
    return qamw.combine(y, r.positions, r.weights)


def build(experts, width, hidden, seed=0, device="cuda"):
    """A layer's matrices, synthetic: (router [experts][width] bf16, up, down) with the experts decoded to bf16."""
    up = torch.stack([synth.weight_device(seed + 2 * e, 2 * hidden, width, 1.0, "bf16") for e in range(experts)])
    down = torch.stack([synth.weight_device(seed + 2 * e + 1, width, hidden, 1.0, "bf16") for e in range(experts)])
    gen = torch.Generator(device=device).manual_seed(seed)
    router = (torch.randn(experts, width, generator=gen, device=device) / width**0.5).bfloat16()
    return router, stored_and_decoded(up), stored_and_decoded(down)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--choices", type=int, default=2)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=1024)
    a = ap.parse_args()
    router, up, down = build(a.experts, a.width, a.hidden)
    up8, down8 = in_8_bits(up), in_8_bits(down)
    x = torch.randn(a.tokens, a.width, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    logits = x @ router.t()
    results = {}
    for name, u, d in (("bf16", up, down), ("8 bits", up8, down8)):
        for _ in range(3):
            results[name] = routed_layer(x, logits, u, d, a.choices)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()                              # a pass is up to six launches: captured once, replayed with one
        with torch.cuda.graph(graph):
            held = routed_layer(x, logits, u, d, a.choices)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, results[name])
        t = time.perf_counter()
        for _ in range(20):
            graph.replay()
        torch.cuda.synchronize()
        size = sum(e.weights.numel() * e.weights.element_size() for e in (u, d))
        print(f"{name}: {(time.perf_counter() - t) / 20 * 1e6:.0f} us a pass, {size / 1e6:.0f} MB of weights")
    off = (results["8 bits"].float() - results["bf16"].float()).norm() / results["bf16"].float().norm()
    print(f"8 bits against bf16: relative difference {off:.4f}")
    return float(off)


if __name__ == "__main__":
    main()
