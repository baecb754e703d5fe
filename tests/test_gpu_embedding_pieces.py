"""Embedding gradients of so many tokens that a group of lanes goes through 16, 32 or 64 sorted positions, and the lookup and
the gradient of more bytes than the last-level cache keeps.  A sum of c rows has at most c + 1 roundings of 2^-24 against the
sum of absolute values and the scale's, as in test_gpu_embedding."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
from oracle import operators_oracle as O
from test_gpu_embedding import bits, tokens

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def piece_of(n, D):
    """Positions of a group of lanes, by the rule of the library: 8 while that fills the chip, up to 64."""
    lanes = 8
    while lanes < (D + 7) // 8 and lanes < 256:
        lanes *= 2
    piece = 8
    while piece < 64 and n * lanes // 256 >= 1024 * piece:
        piece *= 2
    return piece


def check(ids, V, D, dtype, out_dtype, accumulate, scale=1.5, seed=0):
    n = len(ids)
    gen = torch.Generator().manual_seed(seed + n + D)
    g = torch.randn((n, D), generator=gen).to(dtype)
    old = torch.randn((V, D), generator=gen).to(out_dtype)
    table = old.cuda() if accumulate else torch.full((V, D), float("nan"), dtype=out_dtype, device="cuda")
    ws = torch.empty(P.sv_embedding_grad_workspace_bytes(n, V, D), dtype=torch.uint8, device="cuda").fill_(255)
    P.sv_embedding_grad(g.cuda(), ids.cuda(), table, scale, accumulate, ws)
    got = O.values(bits(table))
    given = ((ids >= 0) & (ids < V)).numpy()
    key = np.where(given, ids.numpy(), V)
    order = np.argsort(key, kind="stable")
    present, start, c = np.unique(key[order], return_index=True, return_counts=True)
    touched = present[present < V]
    for j, v in enumerate(touched):
        rows = O.values(bits(g[torch.from_numpy(order[start[j]:start[j] + c[j]])]))
        s, a = rows.sum(0) * scale, np.abs(rows).sum(0) * scale
        if accumulate:
            o = O.values(bits(old[v]))
            s, a = s + o, a + np.abs(o)
        tol = (c[j] + 2) * 2.0 ** -24 * a + 2.0 ** -24 * np.abs(s) + 1e-38
        assert O.within(got[v], s, tol, out_dtype == BF16).all(), (v, c[j])
    rest = np.setdiff1d(np.arange(V), touched)
    if accumulate:
        assert np.array_equal(bits(table)[rest], bits(old)[rest])
    else:
        assert not got[rest].any()                       # (NaN counts)
    return table


def counted(n, piece, V, seed):
    """n tokens: counts about a piece and about several, tokens of one position, and the rest of two tokens and of none."""
    counts = [piece - 1, piece, piece + 1, 1, 2 * piece - 1, 1, 1, 2 * piece, 2 * piece + 1, 3 * piece, 1, piece // 2, 5 * piece + 3, 40 * piece + 1,
              piece, piece, 1, piece - 2, 1, 63, 64, 65, 127, 128, 129, 7, 8, 9]
    ids = np.repeat(np.arange(len(counts)), counts)
    left = n - len(ids)
    assert left > 100 and V > len(counts) + 400
    rng = np.random.default_rng(seed)
    some = rng.integers(len(counts) + 2, V - 2, size=left // 3)
    ids = np.concatenate([ids, some, np.full(left // 4, len(counts)), np.full(50, -1), np.full(30, V), np.full(20, -7)])
    ids = np.concatenate([ids, np.full(n - len(ids), len(counts) + 1)])
    return torch.from_numpy(rng.permutation(ids).astype(np.int32))


# lanes of a row: 256, 256, 128, 8 (32 groups to a workgroup)
@pytest.mark.parametrize("piece, n, D", [(8, 8191, 1027), (16, 8192, 1027), (16, 16383, 1032), (32, 16390, 1027), (64, 32769, 1027),
                                         (64, 65601, 520), (16, 262144, 3), (32, 524309, 8), (64, 1048600, 5)])
@pytest.mark.parametrize("dtype, out_dtype, accumulate", [(F32, F32, False), (BF16, BF16, True), (BF16, F32, False), (F32, BF16, True)])
def test_pieces(piece, n, D, dtype, out_dtype, accumulate):
    assert piece_of(n, D) == piece
    check(counted(n, piece, 601, n), 601, D, dtype, out_dtype, accumulate)


@pytest.mark.parametrize("kind", ["one", "uniform", "zipf"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_long_pieces_of_other_distributions(kind, accumulate):
    n, V, D = 33001, 3001, 1040
    assert piece_of(n, D) == 64
    check(tokens(n, V, 3, kind), V, D, BF16, BF16, accumulate)


@pytest.mark.parametrize("dtype, D", [(BF16, 2056), (F32, 1030)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_past_the_cache(dtype, D, accumulate):
    n, V = 33000, 700
    assert n * D * (4 if dtype == F32 else 2) > 128 << 20
    check(counted(n, 64, V, 1), V, D, dtype, F32, accumulate)


def test_the_same_bits_every_time():
    ids = counted(33000, 64, 601, 2)
    a = [check(ids, 601, 1027, BF16, F32, False) for _ in range(2)]
    assert torch.equal(a[0], a[1])


@pytest.mark.parametrize("dtype, n, D", [(BF16, 33000, 1027), (F32, 9001, 2048), (BF16, 1200001, 40)])
def test_lookup_past_the_cache(dtype, n, D):
    V = 501
    assert 2 * n * D * (4 if dtype == F32 else 2) > 128 << 20
    w = torch.randn((V, D), generator=torch.Generator().manual_seed(D)).to(dtype).cuda()
    ids = tokens(n, V, n).cuda()
    out = torch.full((n, D), 9.0, dtype=dtype, device="cuda")
    flags = torch.full((n,), 9, dtype=torch.int32, device="cuda")
    P.sv_embedding(w, ids, out, 0.75, flags)
    ok = (ids >= 0) & (ids < V)
    want = torch.where(ok[:, None], w.index_select(0, torch.where(ok, ids, 0)).float() * 0.75, 0.0).to(dtype)
    assert torch.equal(out, want)
    assert torch.equal(flags, torch.where(ok | (ids == -1), 0, 16).int())
