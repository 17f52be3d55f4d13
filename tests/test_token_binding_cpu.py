"""What the binding of the losses over given tokens decides without a device."""
import itertools

import pytest

from paper_1804_06087_amd import binding as bd


@pytest.mark.parametrize("n", [1, 2, 3, 5])
def test_rows_overlap(n):
    """Against the bytes themselves: two matrices of n rows of `width` bytes, at every offset."""
    width = 4
    for ld_p, ld_q in itertools.product((0, 1, 3, 4, 5, 8, 9, 12, 16), repeat=2):
        for q in range(0, 120):
            p = 60
            bytes_p, bytes_q = ({first + i * ld + k for i in range(n) for k in range(width)} for first, ld in ((p, ld_p), (q, ld_q)))
            assert bd._rows_overlap(p, ld_p, q, ld_q, n, width) == bool(bytes_p & bytes_q), (ld_p, ld_q, q)


def test_rows_overlap_of_many_rows():
    """More rows than are looked at together."""
    n = (1 << 20) + 7
    assert not bd._rows_overlap(0, 16, 8, 32, n, 8)
    assert bd._rows_overlap(0, 16, 8, 31, n, 8)
    assert bd._rows_overlap(0, 1 << 30, (n - 1 << 30) + 4, 8, n, 8)
    assert not bd._rows_overlap(0, 1 << 30, (n - 1 << 30) + 8, 8, n, 8)
