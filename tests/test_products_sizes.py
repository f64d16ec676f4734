"""Stacks too large to be numbered in 32 bits (no GPU)."""
import ctypes

import pytest

import paper_2512_22492_gb300 as rr
from paper_2512_22492_gb300.products import _Quant
from paper_2512_22492_gb300.rr import _lib

LARGEST = 2 ** 31 - 1


def sizes(rows, cols, count, group, pair):
    c = _Quant(rows, cols, count, group, 0, pair)
    one, total = ctypes.c_int64(-7), ctypes.c_int64(-7)
    return _lib.rr_quant_bytes(ctypes.byref(c), ctypes.byref(one), ctypes.byref(total)), one.value, total.value


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("rows,cols,count,pair", [
    (LARGEST, 1 << 18, 65535, 0), (LARGEST - 1, 1 << 18, 65535, 1), (LARGEST, 1 << 18, 1, 0),
    (LARGEST, 129, 17, 0), (1 << 20, 1 << 18, 16, 0)])
def test_too_many_blocks_are_refused(rows, cols, count, pair, group):
    """Not a size that has wrapped round 64 bits."""
    with pytest.raises(rr.RRError, match="RR_ELAYOUT.*blocks"):
        rr.Quantized(rows, cols, group, "bf16", bool(pair), count, data=None)
    status, one, total = sizes(rows, cols, count, group, pair)
    assert status != 0 and one == total == -7


@pytest.mark.parametrize("rows,cols,count,pair,blocks", [
    (LARGEST, 128, 15, 0, 15 * 2 ** 27), (1 << 20, 1 << 18, 15, 0, 15 * 2 ** 27),
    (16, 128, 65535, 0, 65535), (LARGEST - 1, 1, 15, 1, 15 * 2 ** 27)])
def test_the_largest_stacks(rows, cols, count, pair, blocks):
    status, one, total = sizes(rows, cols, count, 32, pair)
    assert status == 0 and total == 1152 * blocks and one * count == total
