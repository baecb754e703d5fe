"""More rows or tokens than one launch has workgroups for (a launch has fewer than 2^32 lanes), with rows so short that
they fit: 2^24 workgroups of 256 lanes are the first too many."""
import pytest
import torch

import paper_2509_24328_amd as P

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
N = (1 << 24) + 5


@pytest.fixture(scope="module")
def rows():
    """Logits of two entries, tokens (-1, 0, 1), and the log-probabilities by definition."""
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB")
    gen = torch.Generator(device="cuda").manual_seed(3)
    z = (2 * torch.randn((N, 2), generator=gen, device="cuda")).to(BF16)
    tok = torch.randint(-1, 2, (N,), generator=gen, device="cuda", dtype=torch.int32)
    tok[-5:] = 1
    lp = torch.log_softmax(z.double(), -1)
    want = torch.where(tok < 0, 0.0, lp.gather(1, tok.clamp(min=0).long()[:, None])[:, 0])
    return z, tok, lp, want


def test_rows_scored(rows):
    z, tok, lp, want = rows
    logprob, rank = torch.full((N,), 9.0, device="cuda"), torch.full((N,), 9, dtype=torch.int32, device="cuda")
    P.sv_token_logprobs(z, tok, logprob, rank=rank)
    assert ((logprob - want).abs() <= 2e-6 + 1.3e-7 * want.abs()).all()
    other = z.float().flip(1).gather(1, tok.clamp(min=0).long()[:, None])[:, 0]
    own = z.float().gather(1, tok.clamp(min=0).long()[:, None])[:, 0]
    first = (other > own) | ((other == own) & (tok == 1))
    assert torch.equal(rank, torch.where(tok < 0, 0, 1 + first.int()).int())


def test_packed_rows_scored(rows):
    """One sequence after the other in z, of five positions at most, the last ones in the second launch."""
    z, tok, lp, want = rows
    B, Pn = (N + 4) // 5 + 1, 5
    count = torch.full((B,), 5, dtype=torch.int64, device="cuda")
    count[-2], count[-1] = N - 5 * (B - 2), 0
    offs = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), count.cumsum(0)]).int()
    assert int(offs[-1]) == N and B * Pn > (1 << 24)
    tokens = torch.full((B * Pn,), 1, dtype=torch.int32, device="cuda")
    tokens[:N] = tok
    logprob = torch.full((B * Pn,), 9.0, device="cuda")
    P.sv_token_logprobs(z, tokens.view(B, Pn), logprob.view(B, Pn), t_offsets=offs)
    assert ((logprob[:N] - want).abs() <= 2e-6 + 1.3e-7 * want.abs()).all()
    assert not logprob[N:].any()


def test_gradients_of_rows(rows):
    z, tok, lp, want = rows
    g = torch.full((N,), 2.0, device="cuda")
    logprob, dz = torch.full((N,), 9.0, device="cuda"), torch.full((N, 2), 9.0, dtype=F32, device="cuda")
    z = z.float()
    P.sv_token_logprobs_grad(z, tok, g, dz, logprob=logprob)
    assert ((logprob - want).abs() <= 2e-6 + 1.3e-7 * want.abs()).all()
    one = torch.nn.functional.one_hot(tok.clamp(min=0).long(), 2)
    ref = torch.where((tok < 0)[:, None], 0.0, 2 * (one - lp.exp()))
    # a probability is off by 2.5e-6 of itself and 1.3e-7 / ln 2 for each nat of distance, weighted with 2; the token's 2 and the result are rounded
    tol = 2 * lp.exp() * (2.5e-6 + 1.3e-7 / 0.69 * lp.abs()) + 2 * 2.4e-7 * one + 2.4e-7 * ref.abs() + 1e-36
    assert ((dz - ref).abs() <= tol).all()


def test_rows_of_a_table():
    """2^29 tokens of one column: 32 rows to a workgroup."""
    n, V = (1 << 29) + 7, 1000
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    gen = torch.Generator(device="cuda").manual_seed(5)
    table = torch.randn((V, 1), generator=gen, device="cuda").to(BF16)
    ids = torch.randint(0, V, (n,), generator=gen, device="cuda", dtype=torch.int32)
    ids[-3], ids[-2] = -1, V
    out = torch.full((n, 1), 9.0, dtype=BF16, device="cuda")
    flags = torch.full((n,), 9, dtype=torch.int32, device="cuda")
    P.sv_embedding(table, ids, out, flags=flags)
    padded = torch.cat([table, torch.zeros((1, 1), dtype=BF16, device="cuda")])
    for i in range(0, n, 1 << 27):
        k = ids[i:i + (1 << 27)]
        k = torch.where((k >= 0) & (k < V), k, V)
        assert torch.equal(out[i:i + (1 << 27), 0], padded[:, 0].index_select(0, k)), i
    assert flags[-3] == 0 and flags[-2] == 16 and int((flags != 0).sum()) == 1


def test_positions_of_long_rows():
    """512 lanes to a position: 2^23 are the first too many.  Only the last three have a row."""
    B, V = (1 << 23) + 5, 20000
    gen = torch.Generator(device="cuda").manual_seed(7)
    z = torch.randn((3, V), generator=gen, device="cuda")
    offs = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    offs[-3:] = torch.tensor([1, 2, 3], dtype=torch.int32)
    tok = torch.full((B, 1), 11, dtype=torch.int32, device="cuda")
    logprob, top = torch.full((B, 1), 9.0, device="cuda"), torch.full((B, 1, 1), 9, dtype=torch.int32, device="cuda")
    val = torch.full((B, 1, 1), 9.0, device="cuda")
    P.sv_token_logprobs(z, tok, logprob, top_token=top, top_logprob=val, t_offsets=offs)
    want = torch.log_softmax(z.double(), -1)
    assert ((logprob[-3:, 0] - want[:, 11]).abs() <= 2e-6 + 1.3e-7 * want[:, 11].abs()).all()
    assert torch.equal(top[-3:, 0, 0], z.argmax(-1).int())
    assert not logprob[:-3].any() and (top[:-3] == -1).all() and (val[:-3] == -float("inf")).all()
