"""The zeros of sv_embedding_grad's table, which the launches of the sort write in shares: all of them, for tables whose
bytes are and are not a whole number of shares.  The launches are 2 for V < 512, 4 below 262144 and 6 from there on."""
import pytest
import torch

import paper_2509_24328_amd as P

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
LEAST = 128 << 10                                        # bytes of which a share is a multiple


# (the first three of each type: a few bytes above a multiple of launches x 128 KiB)
@pytest.mark.parametrize("dtype, V, D", [
    (BF16, 4033, 65), (BF16, 15489, 897), (BF16, 52429, 5), (BF16, 4096, 64), (BF16, 511, 513), (BF16, 700, 3),
    (F32, 266177, 65), (F32, 393217, 1), (F32, 262147, 3), (F32, 32768, 4), (F32, 32769, 4), (F32, 511, 257)])
@pytest.mark.parametrize("n", [300, 5000])
def test_every_row_without_a_token_is_zeros(dtype, V, D, n):
    """The last tokens of the table do not occur, and what was there before is NaN."""
    gen = torch.Generator().manual_seed(V)
    ids = torch.randint(0, V // 2, (n,), generator=gen, dtype=torch.int32).cuda()
    g = torch.randint(-8, 9, (n, D), generator=gen).to(dtype).cuda()
    table = torch.full((V + 1, D), float("nan"), dtype=dtype, device="cuda")     # (a row more: stays as it is)
    ws = torch.empty(P.sv_embedding_grad_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda")
    P.sv_embedding_grad(g, ids, table[:V], ws=ws)
    want = torch.zeros((V, D), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), g.double())
    assert want.abs().max() <= 256                       # whole numbers: exact in either type
    assert torch.equal(table[:V].double(), want)
    assert torch.isnan(table[V]).all()


def test_the_sizes_are_at_the_edge():
    """Some of the tables above are a last element or two more than whole shares."""
    for V, D, size, launches in ((4033, 65, 2, 4), (15489, 897, 2, 4), (52429, 5, 2, 4), (266177, 65, 4, 6), (393217, 1, 4, 6)):
        assert 0 < V * D * size % (launches * LEAST) < launches, (V, D)
