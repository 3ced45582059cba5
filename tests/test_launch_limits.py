"""Products of more tiles than a launch has (2^32 threads) are refused before anything is launched, with the status that the header names."""
import pytest

from paper_2605_26339_amd import qamw

P = 1 << 20                                                     # never followed


@pytest.mark.parametrize("d_out", [(1 << 14) + 1, 1 << 15, 1 << 18, 1 << 24])
@pytest.mark.parametrize("gated", [0, 1])
def test_products_of_any_alignment(d_out, gated):
    """Rows of 8 bytes: 64 x 64 outputs a tile, 2^16 row tiles."""
    m = 1 << 22
    L = qamw.lib()
    rc = L.qamw_int8_matmul(P, qamw.DTYPE_I8, P, None, m, 8, P, P, 8, d_out, 8, gated, P, 1, d_out, None, 0, None)
    assert rc == qamw.ERR_UNSUPPORTED
    rc = L.qamw_grouped_matmul(P, qamw.DTYPE_BF16, None, m, 8, None, P, None, 8, 0, P, 4, m, d_out, 4, gated, P, 1, d_out, None)
    assert rc == qamw.ERR_UNSUPPORTED
