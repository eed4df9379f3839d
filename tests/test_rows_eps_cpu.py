"""A norm's eps that is subnormal in fp32 is refused: the reciprocal root takes such a number for 0, and a row of zeros would become NaN."""
import pytest

import paper_2604_05250_amd as dd

A, SHAPE = 1 << 20, -2


@pytest.mark.parametrize("eps", [1e-39, 1.1754942e-38, 1.4e-45])
@pytest.mark.parametrize("side", ["queries", "keys", "pages"])
def test_subnormal_eps(side, eps):
    st = (2 * 5 * 64, 5 * 64, 64)
    if side == "pages":
        rc = dd.lib().dd_paged_cache_append(A, 2 * A, None, None, 3 * A, *st, 4 * A, *st, 5 * A, 6 * A, None, None, 7 * A, eps, None, 0, 0, 5, 2, 2, 64, 9, 16, 4,
                                            dd.BF16, dd.BF16, None)
    else:
        weights = (7 * A, None) if side == "queries" else (None, 7 * A)
        rc = dd.lib().dd_qk_norm_rope(A, *st, 2 * A, *st, *weights, eps, None, 0, 0, None, 3 * A, 4 * A, 2, 2, 2, 5, 64, dd.BF16, None)
    assert rc == SHAPE
