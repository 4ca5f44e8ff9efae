"""Sizes near the end of 32 bits are refused before any device is touched (CPU)."""
import ctypes

import pytest

import paper_2306_17266_b200 as sgs

EINVAL, EUNSUPPORTED = sgs.binding.SGS_EINVAL, sgs.binding.SGS_EUNSUPPORTED
P = 1 << 20  # an address that is never read: no device owns it


@pytest.mark.parametrize("dtype", [sgs.SGS_BF16, sgs.SGS_F32])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("sides", ["row", "col", "both"])
@pytest.mark.parametrize("rows,cols,status", [(2 ** 31 - 1, 1, EUNSUPPORTED), (2 ** 31 - 64, 1, EUNSUPPORTED), (2 ** 31 - 128, 1, EUNSUPPORTED),
                                              (2 ** 31 - 512, 1, EUNSUPPORTED), (1, 2 ** 31 - 100, EUNSUPPORTED), (5, 2 ** 31 - 1, EUNSUPPORTED),
                                              (2 ** 31 - 513, 1, EINVAL), (1, 2 ** 31 - 513, EINVAL)])  # (the largest sizes taken: the address is what is wrong)
def test_quantize_near_the_end_of_32_bits(rows, cols, status, sides, block_rows, dtype):
    d = sgs.QuantizeF8Desc(rows=rows, cols=cols, dtype=dtype, block_rows=block_rows, ldq=cols, ldqt=rows)
    row, col = (P if sides != "col" else None), (P if sides != "row" else None)
    assert sgs.lib().sgs_quantize_f8(ctypes.byref(d), P, row, row, col, col, None) == status
