"""Rows as long as the entry points take them, where a column's number no longer leaves room above it in 32 bits."""
import pytest
import torch

from paper_2605_26339_amd import qamw

from .test_served_layers import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
LONGEST = 2**31 - 1


@pytest.mark.parametrize("d", [LONGEST, LONGEST - 6, LONGEST - 7])
def test_combine_of_the_longest_rows(d):
    """One row with a weight of 1: the row itself, and nothing behind it."""
    say(f"[combine] a row of {d}")
    y = torch.full((1, d + 9), float("nan"), dtype=torch.bfloat16, device=DEV)
    y[:, :d].uniform_(generator=torch.Generator(DEV).manual_seed(1))
    out = torch.full((1, d + 9), 7.0, dtype=torch.bfloat16, device=DEV)
    one = torch.ones(1, 1, device=DEV)
    qamw.combine(y[:, :d], torch.zeros(1, 1, dtype=torch.int32, device=DEV), one, out=out[:, :d])
    assert torch.equal(out[:, :d], y[:, :d]) and (out[:, d:] == 7).all()


@pytest.mark.parametrize("d", [LONGEST])
def test_quantise_the_longest_row(d):
    """By the definition, piece by piece; the largest value is the last one, and nothing is written behind it."""
    say(f"[quantise] a row of {d}")
    x = torch.empty(1, d, dtype=torch.bfloat16, device=DEV).uniform_(-1, 1, generator=torch.Generator(DEV).manual_seed(2))
    x[0, -1] = 2.0
    codes = torch.full((1, d + 9), 77, dtype=torch.int8, device=DEV)
    scales = torch.empty(1, device=DEV)
    qamw.int8_quantize(x, out=(codes[:, :d], scales))
    assert scales.item() == torch.tensor(2.0).div(127).item() and (codes[:, d:] == 77).all() and codes[0, d - 1] == 127
    for a in range(0, d, 1 << 28):
        b = min(a + (1 << 28), d)
        assert torch.equal(codes[0, a:b], (x[0, a:b].float() * 63.5).round().to(torch.int8))   # 127 / 2 is exact
