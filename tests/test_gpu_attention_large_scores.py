"""sv_chunk_attention where scores are far beyond 2^24.

Q and k have one column each that is not 0, powers of two times whole numbers below 2^8, so their products are exact, and two different
scores of a row lie more than 2^10 apart: weights are 0 or equal.  Then out is the mean of the values of the row's largest
keys, off by 2^-24 of sum_j w_j |v_j| for each of n products and sums and the division's two, by half a step of its type for the result, and by the
rounding of the weights: 2^-8 of each for bfloat16 queries (a weight is 2^r with r what a score's rounding leaves of it beside the maximum, below 2^24 up
to 1/2: w and not 1 is rounded, while the sum of the weights is not), and 2^-24 for float32 queries over 8-bit caches, whose values' scales are a part of the
weights.  lse is the score and log n, off by 2^-24 of itself for each of the scale's rounding, the product's, lse's own, and less than one more for
the rest: 2^-22."""
import numpy as np
import pytest
import torch

import test_gpu_chunk_attention as A
from test_gpu_chunk_attention import BF16, F8, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [10, 24, 27, 31, 35, 40, 80, 110])
@pytest.mark.parametrize("T, group, D, page", [(1, 1, 64, 16), (3, 4, 128, 16), (9, 4, 72, 20), (5, 2, 256, 32), (40, 4, 64, 16), (70, 2, 120, 12)])
@pytest.mark.parametrize("dtype, kind", TYPES)
def test_scores_of_any_size(dtype, kind, T, group, D, page, power):
    """Scores of about 2^power and of both signs, the largest of them once or several times and in any step of 32 keys."""
    lengths, heads, Hq = [45, 0, 130, 300], 2, 2 * group
    cache, pages = A.make(lengths, [T] * 4, heads, D, page, kind, seed=T, garbage=False)
    g = torch.Generator().manual_seed(power)
    factor = torch.randint(-120, 121, cache.k.shape[:3], generator=g).float()
    if kind == F8:                                       # (whole numbers of four bits, and powers of two for scales)
        factor = torch.randint(-15, 16, cache.k.shape[:3], generator=g).float()
        cache.k_scale.fill_(2.0 ** (power // 2))
        cache.k.copy_((factor[..., None] * (torch.arange(D) == 3)).to(F8).cuda())
    else:
        cache.k.copy_((factor[..., None] * (torch.arange(D) == 3) * 2.0 ** (power // 2)).to(kind).cuda())
    q = torch.zeros((4 * T, Hq, D), dtype=dtype, device="cuda")
    sign = (torch.randint(0, 2, (4 * T, Hq), generator=g) * 2 - 1).float()
    q[..., 3] = (sign * 2.0 ** (power - power // 2)).to(dtype).cuda()
    out, lse, flags = A.run(cache, q.view(4, T, Hq, D), lengths, pages, None, None, scale=0.125)
    out, lse = out.double().cpu().numpy().reshape(-1, Hq, D), lse.double().cpu().numpy().reshape(-1, Hq)
    assert (flags == 0).all()
    k, v = A.held(cache)
    qd = q.cpu().double().numpy()
    for r in range(4 * T):
        b, p = r // T, lengths[r // T] + r % T
        pg, sl = pages[b, np.arange(p + 1) // page].numpy(), np.arange(p + 1) % page
        for h in range(Hq):
            s = 0.125 * qd[r, h, 3] * k[pg, h // group, sl, 3]
            w = (s == s.max()).astype(float)
            n, values = w.sum(), v[pg, h // group, sl]
            if power == 10:                              # (apart by 2^7 at least: e^-128 is nothing either)
                assert s.max() - s[s < s.max()].max(initial=-np.inf) >= 2.0 ** 7
            ref, wabs = w @ values / n, w @ np.abs(values) / n
            half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
            tol = ((len(s) + 2) * 2.0 ** -24 + (half if kind == F8 or dtype == BF16 else 0.0)) * wabs + half * np.abs(ref)
            assert (np.abs(out[r, h] - ref) <= tol * (1 + 1e-6)).all(), (r, h, np.abs(out[r, h] - ref).max())
            want = s.max() + np.log(n)
            assert abs(lse[r, h] - want) <= 2.0 ** -22 * abs(want) + 2.0 ** -22, (r, h, lse[r, h], want)
