"""sv_chunk_attention with more row blocks than a launch holds."""
import pytest
import torch

import paper_2509_24328_amd as P
from test_gpu_chunk_attention import BF16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("B, heads", [(2 ** 24 + 77, 1), (2 ** 21 + 3, 9)])
def test_more_row_blocks_than_a_launch(B, heads, packed):
    """Sequences of one token that see it alone, or nothing: the value itself, or 0."""
    D, n_pages = 8, 5
    cache = P.Cache.empty(n_pages, heads, 1, D, BF16)
    g = torch.Generator().manual_seed(0)
    cache.k.copy_(torch.randn(cache.k.shape, generator=g))
    cache.v.copy_(torch.randn(cache.v.shape, generator=g))
    number = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    table = (number[:B] % n_pages)[:, None].contiguous()
    first = (number[:B] % 7 == 3).int()
    q = torch.ones((B, heads, D) if packed else (B, 1, heads, D), dtype=BF16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:-1], 7.0, device="cuda")
    flags = torch.full((B,), 9, dtype=torch.int32, device="cuda")
    P.sv_chunk_attention(cache, q, out, torch.zeros(B, dtype=torch.int32, device="cuda"), table, t_offsets=number if packed else None,
                         P=1 if packed else None, first=first, lse=lse, flags=flags)
    want = cache.v[table[:, 0].long()][:, :, 0] * (1 - first)[:, None, None].to(BF16)
    assert torch.equal(out.view(want.shape), want) and (flags == 0).all()
    assert torch.equal(torch.isinf(lse.view(B, heads)), (first == 1)[:, None].expand(B, heads))
