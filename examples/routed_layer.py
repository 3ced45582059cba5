"""A routed feed-forward layer served from packed experts.

Every expert's matrices are coded by the codec, as they would be stored; to serve them they are decoded to bf16 and, for the 8-bit
layer, quantised once more to 8-bit integers with a scale for each output channel, or for the 4-bit one to 4-bit floats with a
scale for every 32 columns.  A pass is: logits to experts, tokens to 8 or 4 bits, the gate and up projections of the chosen experts with
silu(gate) * up, that to 8 or 4 bits, the down projections, and the weighted sum back to the tokens.  `routed_block` has the norms around it,
too, and chooses experts by sigmoid scores with a bias, from the best groups.

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


def in_4_bits(experts):
    """The same experts in 4-bit floating point."""
    n, outs, ins = experts.weights.shape
    q = qamw.mx4_quantize(experts.weights.view(n * outs, ins))
    return qamw.Mx4(q.codes.view(n, outs, -1), q.scales.view(n, outs, -1), ins)


def routed_block(h, norm_weight, router, bias, up, down, choices, groups, top_groups, next_weight, gate=None):
    """A block in 4 bits with the norms around it: h [tokens][width] bf16 is the stream, router [experts][width], bias [experts] fp32, up
    and down as routed_layer takes them.  Returns the stream after the block and, in 4 bits, the norm of it that the next block takes."""
    _, x = qamw.block_norm(h, norm_weight)
    r = qamw.route_scored(x @ router.t(), choices, bias=bias, groups=groups, top_groups=top_groups)
    y = experts_in_4_bits(x, r, up, down)
    return qamw.block_norm(h, next_weight, block=y, gate=gate, quantize="mx4")


def experts_in_4_bits(x, r, up, down):
    h = qamw.mx4_grouped_matmul(x, up, r.offsets, rows=r.rows, gated=True)      # the tokens once, however many experts they have
    return qamw.combine(qamw.mx4_grouped_matmul(h, down, r.offsets), r.positions, r.weights)


def routed_layer(x, logits, up, down, choices):
    """x [tokens][width] bf16, logits [tokens][experts]; up [n][2 hidden][width] (gates, then up projections), down [n][width][hidden],
    both in 4 bits, in 8 bits or in bf16.  Returns [tokens][width] bf16."""
    r = qamw.route(logits, choices)
    if isinstance(up, qamw.Mx4):
        return experts_in_4_bits(x, r, up, down)
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
    up8, down8, up4, down4 = in_8_bits(up), in_8_bits(down), in_4_bits(up), in_4_bits(down)
    x = torch.randn(a.tokens, a.width, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    logits = x @ router.t()
    results = {}
    for name, u, d in (("bf16", up, down), ("8 bits", up8, down8), ("4 bits", up4, down4)):
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
        size = sum(e[0].numel() * e[0].element_size() for e in (u, d))
        print(f"{name}: {(time.perf_counter() - t) / 20 * 1e6:.0f} us a pass, {size / 1e6:.0f} MB of weights")
    off = {}
    for name in ("4 bits", "8 bits"):
        off[name] = float((results[name].float() - results["bf16"].float()).norm() / results["bf16"].float().norm())
        print(f"{name} against bf16: relative difference {off[name]:.4f}")
    return off["8 bits"]


if __name__ == "__main__":
    main()
