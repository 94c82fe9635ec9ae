"""Host-only checks of the byte ranges that the bf16 products' loads are held
to: every load of a tile that lies in its operand's range lies in the matrix
itself, also where that is the right-hand columns of a wider one and ends its
allocation, and no element that a product needs is out of range."""
import ctypes

import pytest

from paper_2510_14614_amd import fal

TILES = (64, 128, 256)


def span(kmaj, ld, r0, rows, k):
    f = fal.lib().fal_gemm_operand_bytes
    f.restype = ctypes.c_int64
    f.argtypes = [ctypes.c_int32, ctypes.c_int64] + [ctypes.c_int32] * 3
    return f(kmaj, ld, r0, rows, k)


# rows of the output dimension, stride, k-rows: dense; halves of one matrix and
# narrower slices of a wider one, whose rows fill no whole tile
SLICES = [(128, 128, 64), (120, 240, 64), (1000, 2000, 1024), (2752, 5504, 8192), (10944, 21888, 8192), (8, 16, 1),
          (72, 1000, 33), (1000, 1024, 1501), (2744, 2768, 5), (200, 1 << 20, 3)]


@pytest.mark.parametrize("rows,ld,k", SLICES)
def test_strided_operands_end_with_their_last_element(rows, ld, k):
    last = (k - 1) * ld + rows  # elements from the matrix's first to its last
    for tile in TILES:
        for r0 in range(0, rows, tile):
            nbytes = span(0, ld, r0, rows, k)
            # a lane's 16 bytes at column c of a k-row are loaded if they begin inside
            # the range, which is a whole number of them: none pass the last element
            assert nbytes % 16 == 0 and 2 * r0 + nbytes <= 2 * last
            # ... and the last k-row's columns up to the last one are inside
            assert nbytes >= 2 * ((k - 1) * ld + rows - r0)
            # k-rows past the end read as zeros
            assert nbytes <= 2 * k * ld


def test_rows_that_are_no_whole_chunks():
    """50257 columns in rows of 50264 (a vocabulary): the last chunk is read
    whole, inside its row."""
    assert span(0, 50264, 0, 50257, 100) == 100 * 50264 * 2
    assert span(0, 60000, 128, 50257, 100) == (99 * 60000 + 50264 - 128) * 2


@pytest.mark.parametrize("rows,ld,k", SLICES)
def test_contiguous_operands_end_with_their_last_row(rows, ld, k):
    # (columns past k are masked lane by lane)
    for r0 in range(0, rows, 128):
        assert span(1, ld, r0, rows, k) == (rows - r0) * ld * 2
