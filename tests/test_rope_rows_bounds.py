"""Rows of the rotation table at the ends of what a call may ask for."""
import numpy as np
import pytest

from paper_2101_01321_b200 import binding

ARG = -1


@pytest.fixture(scope="module")
def rows_of():
    from paper_2101_01321_b200 import build
    build.build()

    def call(f, pos0, n):
        rows = np.full((max(n, 1), 2 * f.size), 77, np.int16)
        return binding.lib().ibert_rope_rows(f.ctypes.data, 2 * f.size, pos0, n, 1.0, rows.ctypes.data), rows

    return call


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_angles_past_the_range_are_refused(rows_of, sign):
    """A finite frequency times a position may still overflow: it has no cosine, and no row is written."""
    f = np.full(8, 1e-3)
    f[5] = sign * 1e308
    for pos0, n in ((1 << 40, 1), (0, 3)):
        code, rows = rows_of(f, pos0, n)
        assert code == ARG and (rows == 77).all()
    code, rows = rows_of(f, 0, 2)                       # positions 0 and 1: finite
    assert code == 0 and np.abs(rows).max() <= 16384
    assert rows_of(f, 1 << 40, 0)[0] == 0


def test_positions_past_63_bits_are_refused(rows_of):
    f = np.full(8, 1e-3)
    last = (1 << 63) - 1
    code, rows = rows_of(f, last, 2)
    assert code == ARG and (rows == 77).all()
    assert rows_of(f, last, 1)[0] == 0 and rows_of(f, last - 1, 2)[0] == 0 and rows_of(f, last, 0)[0] == 0
