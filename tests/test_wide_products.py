"""The products of many rows, whose workgroups go from tile to tile: bit for bit against sums in 64 bits in int8, within the bound of the
roundings in bf16.  Sums of whole numbers below 2^53 are exact in 64 bits, on the device as on the CPU."""
import math

import numpy as np
import pytest
import torch

from paper_2605_26339_amd import qamw

from .test_served_layers import _strided, check, gate_ref, say

gpu = pytest.mark.gpu
DEV = "cuda"
TYPES = (torch.float32, torch.bfloat16)


def _gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _codes(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int32).to(torch.int8)


def _scales(g, *shape):
    """Of different sizes, so that another row's or another output's is not taken for its own; a gate stays below 80 in size with them."""
    return torch.exp(torch.randn(*shape, generator=g, device=DEV).clamp(-1.5, 1.5)) / 127


def _offsets(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def _sums(x, w):
    return torch.mm(x.double(), w.double().t().contiguous())


def _scaled(x, xs, w, ws):
    """The exact sums, then the two prescribed fp32 products."""
    return _sums(x, w).float() * xs[:, None] * ws[None, :]


def expect(got, ref, gated, slack, what):
    """got [m][d_out] against ref [m][outs]: the same bits where nothing but the prescribed steps lies between."""
    if not gated and slack is None:
        assert torch.equal(got, ref.to(got.dtype)), f"{what}: {int((got != ref.to(got.dtype)).sum())} of {got.numel()}"
        return
    want, off = ref.double(), torch.zeros_like(ref, dtype=torch.float64) if slack is None else slack
    if gated:
        h = ref.shape[1] // 2
        want, off = gate_ref(want[:, :h], want[:, h:], off[:, :h], off[:, h:])
    check(got, want.cpu(), off.cpu(), what)


# ---- few columns: a tile is one or two stages, and its scales follow the last one's at once -------------------------------------------


@gpu
@pytest.mark.parametrize("d_in", [16, 128, 144, 256, 272])
@pytest.mark.parametrize("m,d_out,gated", [(8192, 4096, False), (5000, 9001, False), (4100, 4100, False), (4096, 11008, True), (2040, 8184, True)])
def test_int8_of_few_columns(m, d_out, d_in, gated):
    """Two, three and five tiles a workgroup."""
    say(f"[wide] {m} x {d_out} x {d_in} gated {gated}")
    g = _gen(m + d_out + d_in)
    outs = d_out * (2 if gated else 1)
    x, w, xs, ws = _codes(g, m, d_in), _codes(g, outs, d_in), _scales(g, m), _scales(g, outs) / d_in**0.5
    ref = _scaled(x, xs, w, ws)
    for dtype in TYPES:
        y = qamw.int8_matmul(x, w, ws, x_scales=xs, gated=gated, out_dtype=dtype)
        expect(y, ref, gated, None, dtype)


@gpu
@pytest.mark.parametrize("d_in", [16, 144, 256])
@pytest.mark.parametrize("counts,d_out,gated", [([0, 700, 1301, 5, 256, 900, 511, 328], 4112, True), ([0, 700, 1301, 5, 256, 900, 511, 328], 8203, False),
                                                ([150, 90, 129, 231], 16400, False), ([300, 255, 257, 388], 16400, True)])
def test_int8_groups_of_few_columns(counts, d_out, d_in, gated):
    """Experts of uneven numbers of rows, gathered ones."""
    say(f"[wide] {counts} x {d_out} x {d_in} gated {gated}")
    n, m, outs = len(counts), sum(counts), d_out * (2 if gated else 1)
    g = _gen(m + d_out + d_in)
    x, w, xs, ws = _codes(g, m // 2, d_in), _codes(g, n, outs, d_in), _scales(g, m // 2), _scales(g, n, outs) / d_in**0.5
    rows = torch.randint(0, m // 2, (m,), generator=g, device=DEV, dtype=torch.int32)
    off = _offsets(counts)
    for dtype in TYPES:
        y = qamw.grouped_matmul(x, w, off, rows=rows, x_scales=xs, w_scales=ws, gated=gated, out_dtype=dtype)
        for e in range(n):
            a, b = int(off[e]), int(off[e + 1])
            if a < b:
                r = rows[a:b].long()
                expect(y[a:b], _scaled(x[r], xs[r], w[e], ws[e]), gated, None, (dtype, e))
