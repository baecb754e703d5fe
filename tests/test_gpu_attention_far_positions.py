"""sv_chunk_attention at positions beyond 2^30."""
import pytest
import torch

import paper_2509_24328_amd as P
import test_gpu_chunk_attention as A
from test_gpu_chunk_attention import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T, group", [(1, 1), (9, 4), (40, 2)])
@pytest.mark.parametrize("dtype, kind", TYPES)
@pytest.mark.parametrize("page, D", [(65536, 64), (65535, 8)])
def test_positions_beyond_30_bits(dtype, kind, page, D, T, group):
    """The last positions of a long table, most of whose pages are given back: what sv_cache_write stores there is what attention reads, up to
    the last position that there is, 2^31 - 257 - T."""
    last = 2 ** 31 - 257 - T
    for start in (2 ** 30 - 20, 2 ** 30 + 5 * page - 30, last - 60 - T + 1):
        max_pages = start // page + 3
        pages = torch.full((1, max_pages), -1, dtype=torch.int32)
        pages[0, start // page], pages[0, start // page + 1] = 1, 0
        cache = P.Cache.empty(2, 1, page, D, kind)
        g = torch.Generator().manual_seed(T)
        n = 60 + T
        k, v = (torch.randn((1, n, 1, D), generator=g).to(dtype).cuda() for _ in range(2))
        i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
        P.sv_cache_write(cache, k, v, i32([start]), pages.cuda())
        small = P.Cache.empty(-(-n // 16), 1, 16, D, kind)
        table = torch.arange(small.n_pages, dtype=torch.int32)[None]
        P.sv_cache_write(small, k, v, i32([0]), table.cuda())
        q = A.queries(T, group, D, dtype)
        for window in (40, 3):
            got = A.run(cache, q.view(1, T, group, D), [start + 60], pages, None, None, window)
            A.check(small, q, got, [60], table, None, T, window)
            got = A.run(cache, q.view(1, T, group, D), [start + 60], pages, None, None, 0, [start])
            A.check(small, q, got, [60], table, None, T, 0, [0])
    # behind it, nothing is seen
    out, lse, flags = A.run(cache, q.view(1, T, group, D), [last], pages, None, None, 1)
    assert (flags.view(-1)[1:] == 256).all() and torch.isnan(out.view(T, -1)[1:].float()).all() and torch.isnan(lse.view(T, -1)[1:]).all()
