"""sv_chunk_attention with a scale of 0 or next to it: every seen key has the same weight, the output is the mean of the seen values, the
tolerance that of any scores (which are 0)."""
import numpy as np
import pytest
import torch

import test_gpu_chunk_attention as A
from test_gpu_chunk_attention import F8, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-46, float(np.float32(1e-45)), -1e-39])
@pytest.mark.parametrize("T, group, D, page", [(1, 1, 64, 16), (3, 4, 128, 16), (9, 4, 72, 20), (5, 2, 256, 32), (40, 4, 64, 16), (70, 2, 120, 12)])
@pytest.mark.parametrize("dtype, kind", TYPES)
def test_a_scale_of_nothing(dtype, kind, T, group, D, page, scale):
    """The mean of what is seen, with masks that leave parts of steps and rows with nothing, from one row to the staged ones."""
    lengths = [45, 0, 130, 64]
    cache, pages = A.make(lengths, [T] * 4, 2, D, page, kind, seed=T)
    q = A.queries(4 * T, 2 * group, D, dtype)
    exact = float(np.float32(scale))
    for window, first in ((0, None), (24, None), (0, [3, 0, 140, 64]), (50, [46, 500, 0, 0])):
        got = A.run(cache, q.view(4, T, 2 * group, D), lengths, pages, None, None, window, first, scale)
        A.check(cache, q, got, lengths, pages, None, T, window, first, exact)


@pytest.mark.parametrize("T, group", [(6, 2), (40, 4)])
@pytest.mark.parametrize("dtype, kind", TYPES)
def test_a_scale_of_nothing_times_what_is_not_finite(dtype, kind, T, group):
    """0 times an infinity is NaN, in the rows that see the key or have the query."""
    n, at = 45, 45 + 2
    cache, pages = A.make([n], [T], 1, 64, 16, kind)
    q = A.queries(T, group, 64, dtype)
    q[1, 0, 5], q[0, 1, 7] = float("inf"), float("nan")
    pg, sl = pages[0, at // 16].item(), at % 16
    if kind == F8:
        cache.k_scale[pg, 0, sl] = float("nan")
    else:
        cache.k[pg, 0, sl, 1] = float("-inf")
    out, lse, _ = A.run(cache, q, [n], pages, [0, T], T, scale=0.0)
    want = np.zeros((T, group), bool)
    want[2:] = True
    want[1, 0] = want[0, 1] = True
    assert np.array_equal(np.isnan(out.float().cpu().numpy()).all(-1), want)
    assert np.array_equal(np.isnan(lse.cpu().numpy()), want)
    assert np.isfinite(out.float().cpu().numpy()[~want]).all()
