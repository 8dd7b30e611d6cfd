"""Sizes that the orthogonalised update refuses (CPU only: no call here reaches a GPU)."""
import pytest

from paper_1901_08227_b200 import tng

P = 1 << 20                                                 # an address that nobody follows: every call is refused before


@pytest.mark.parametrize("rows,cols", [(4194241, 4194241), (4194241, 5000000), (5000000, 4194241)])
def test_a_shorter_side_beyond_the_grid_is_refused(rows, cols):
    status = tng.lib().tng_orthogonalize(P, tng.F32, 1, rows, cols, cols, 0, 5, 3.4445, -4.775, 2.0315, P, tng.F32, cols, 0, P, None)
    assert status == tng.ERR_INVALID_ARG
