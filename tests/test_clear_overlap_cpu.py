"""Overlap of rows that lie between each other's, through the C ABI with addresses that no
device has: what is refused.  (What is not runs, and is tested on the GPU.)"""
import pytest

from paper_2609_16915_amd import rosetta as R

ALIAS, BF16 = 4, 1
X, OUT = 1 << 40, 2 << 40
FAR = [3 << 40, 4 << 40, 5 << 40]


@pytest.mark.parametrize("rows,dim,xs,at,hs", [
    (4, 64, 128, 2 * 63, 128),       # the last column of x's rows
    (4, 64, 128, 2 * 65, 128),       # the first of its next row
    (4, 64, 127, 2 * 64, 127),       # no room for both in a row
    (4, 64, 128, -2 * 63, 128),      # from before
    (4, 64, 128, 2 * (128 * 3 + 63), 128),   # only the last row
    (4, 64, 128, 2 * 64, 192),       # other distances: by their whole ranges
    (1, 64, 128, 2 * 63, 128),
    ((1 << 31) - 1, 64, 1 << 32, 2 * 63, 1 << 32),  # ranges past 64 bits
])
def test_rows_that_overlap(rows, dim, xs, at, hs):
    st = R.lib().rosetta_rms_norm(X, xs, None, dim, None, BF16, BF16, rows, dim, 1e-5, X + at, hs,
                                  None, dim, None, dim, None, FAR[0], None)
    assert st == ALIAS
