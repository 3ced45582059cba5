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
