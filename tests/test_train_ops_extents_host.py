"""CPU-only: leading dimensions whose matrix spans more than any memory are refused, before the products of extents wrap and the checks for
overlap see a small matrix."""
import pytest

P = 0x10000000                                         # stands for a device address; never dereferenced on the host


@pytest.mark.parametrize("rows,ld", [(2 ** 24 + 1, 2 ** 40), (2 ** 30, 2 ** 40), (2 ** 24, 2 ** 40), (2 ** 22 + 1, 2 ** 40)])
@pytest.mark.parametrize("dt", [0, 1])
def test_wrapping_extents(lgn, rows, ld, dt):
    raw = lgn.raw()
    inside = P + 2 ** 20                               # within the matrix, behind what a wrapped product leaves of it
    assert raw.lgn_fp8_quantize(P, rows, 4, ld, dt, 0, 0, inside, 2 ** 50, None, None, None) == 1
    assert raw.lgn_fp8_matmul(inside, 2 ** 50, 0, 2 ** 51, 2 ** 52, 0, rows, 4, 16, P, ld, dt, 0, None, None) == 1


def test_overlap_far_into_a_large_span(lgn):
    """2^22 rows 2^36 elements apart."""
    raw = lgn.raw()
    inside = P + 2 ** 50
    assert raw.lgn_fp8_quantize(P, 2 ** 22, 4, 2 ** 36, 1, 0, 0, inside, 2 ** 62, None, None, None) == 1
