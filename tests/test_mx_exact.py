"""That the inputs of tests/mx_exact.py are what they are said to be (no GPU)."""
import numpy as np
import pytest

from tests import mx_exact
from tests import mx_reference as ref


@pytest.mark.parametrize("rows,cols", [(1, 1), (40, 100), (96, 64), (131, 70)])
def test_codes_hold_the_values(rows, cols):
    x = mx_exact.held(np.random.default_rng(rows), rows, cols)
    np.testing.assert_array_equal(ref.mx_values(x), x)
    for first in (0, 1, 17, 33):        # blocks along the rows that start anywhere, as an expert's do
        if first < rows:
            np.testing.assert_array_equal(ref.mx_values(x[first:].T), x[first:].T)
    if rows >= 64 and cols >= 64:       # more than one scale
        assert len(np.unique(ref.mx_codes(x)[1])) > 1 and len(np.unique(ref.mx_codes(x.T)[1])) > 1


@pytest.mark.parametrize("M,N,K", mx_exact.LONG)
def test_no_block_is_lost_unseen(M, N, K):
    # every block of 32 of the inner axis, were it left out or its scale another's, changes an output; all sums are exact
    a, b = mx_exact.operands(M, N, K)
    assert K <= mx_exact.MOST_TERMS
    for k in range(0, K, 32):
        part = a[:, k:k + 32].astype(np.float64) @ b[:, k:k + 32].astype(np.float64).T
        assert part.any() and (part == np.rint(part)).all()
