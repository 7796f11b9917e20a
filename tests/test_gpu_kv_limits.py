"""The 4-bit cache at the limits of what it holds: rows that are not finite in long
slots, values up to binary32's range, probabilities of a tree's own nodes, large
offsets and batches, and inputs whose results are exact.  u = 2^-24 as in
test_gpu_kv.py, where the bound on the scores is derived."""
import numpy as np
import pytest

from tests.test_gpu_kv import Both, _rows, oil  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ rows that are not finite
@pytest.mark.parametrize("n", [20, 600, 3000, 40000])
@pytest.mark.parametrize("N,G", [(1, 1), (5, 2), (30, 2)])
def test_not_finite_value_row_reaches_whatever_outweighs_it(oil, n, N, G):  # noqa: F811
    """A value row that is not finite makes the output of every row that sees it NaN,
    also where another position outweighs it by 2^369: in one workgroup (20 rows), in
    a few parts and in many."""
    rng = np.random.default_rng(n + N)
    for bad, top in ((5, n - 3), (n - 3, 5), (n // 2, n - 3)):
        k = np.zeros((2, n, 1, 64), np.float32)
        k[:, top, 0, 0] = 16.0
        v = _rows(rng, 2, n, 1, 64)
        v[1, bad, 0, 7] = np.nan
        c = Both(oil, 2, 1, 64, n)
        c.append(k, v)
        q = np.zeros((2, N, G, 64), np.float32)
        q[..., 0] = 16.0
        out, lse = c.attend(q, scale=1.0)
        assert np.isfinite(out[0]).all() and np.isnan(out[1]).all() and np.isfinite(lse).all()
