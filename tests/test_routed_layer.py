"""The example's routed layer: all operators together, against a plain layer in 64 bits."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("routed_layer_example", os.path.join(ROOT, "examples", "routed_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _plain(x, logits, up, down, k):
    """Token by token, in 64 bits, with the decoded weights; a token without a finite logit gets zeros."""
    out = torch.zeros(x.shape, dtype=torch.float64)
    for t in range(x.shape[0]):
        row = logits[t].double()
        best = sorted((e for e in range(len(row)) if row[e] > -torch.inf), key=lambda e: (-row[e], e))[:k]
        if not best:
            continue
        w = torch.softmax(row[best], 0)
        for e, weight in zip(best, w):
            g, u = (up[e].double() @ x[t].double()).chunk(2)
            out[t] += weight * (down[e].double() @ (g * torch.sigmoid(g) * u))
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,k,width,hidden", [(1, 4, 2, 256, 128), (5, 8, 2, 256, 256), (70, 5, 3, 512, 384), (300, 4, 2, 256, 256)])
def test_routed_layer_against_64_bits(tokens, experts, k, width, hidden):
    print(f"[routed layer] {tokens} tokens, {k} of {experts} experts, {width} x {hidden}", flush=True)
    ex = _example()
    router, up, down = ex.build(experts, width, hidden)
    gen = torch.Generator().manual_seed(tokens)
    x = torch.randn(tokens, width, generator=gen).bfloat16().cuda()
    logits = (x @ router.t()).float()
    if tokens > 4:
        logits[2] = -torch.inf                                      # padding
        logits[3, 1:] = -torch.inf                                  # one expert left
    want = _plain(x.cpu(), logits.cpu(), up.weights.cpu(), down.weights.cpu(), k)
    got = ex.routed_layer(x, logits, up, down, k).cpu().double()
    size = want.norm() / want.numel() ** 0.5
    # bf16: the hidden values, the experts' outputs and the result are rounded to 8 bits of mantissa, 2^-9 each
    assert (got - want).norm() <= 3 * 2.0**-9 * want.norm() + 1e-9
    eight = ex.routed_layer(x, logits, ex.in_8_bits(up), ex.in_8_bits(down), k).cpu().double()
    # 8 bits: a step of max / 127 for inputs, hidden values and both weights; the largest of some hundred normal values is under
    # 5 standard deviations, so a rounding is under 5 / 127 / sqrt(12) = 1.2 % of the size of a value, gate and up both count: 5 of them, and
    # hidden values, products of two, have larger maxima (under 16): 4 % more
    assert (eight - want).norm() <= (5 * 0.012**2 + 0.04**2) ** 0.5 * 1.5 * want.norm() + 1e-9
    if tokens > 4:
        assert (got[2] == 0).all() and (eight[2] == 0).all() and got[3].abs().max() > 0.01 * size
