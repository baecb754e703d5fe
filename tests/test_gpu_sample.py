"""sv_sample against the fp64 definition.

Weights and sums are fp64 on both sides, 1e-12 of the mass apart at most over 2^18 entries: the token is the oracle's wherever no decision
of it lies nearer than that to its other outcome (and such rows are rare: the tests' inputs have none, or say how many).  A log-probability is that
of the token to half a float32 step, and 1e-12."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
from oracle import model_side_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def logits(rows, V, dtype, seed, spread=2.5, pad=0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((rows, V + pad), generator=g) * spread + 8.0 * (torch.rand((rows, V + pad), generator=g) < 0.01)
    return z.to(dtype).cuda()[:, :V], torch.rand(rows, generator=g, dtype=torch.float64).cuda()


def run(z, u, **kw):
    rows = z.shape[0]
    token = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    logprob = torch.full((rows,), 9.0, device="cuda")
    flags = torch.full((rows,), 9, dtype=torch.int32, device="cuda")
    P.sv_sample(z, u, token, logprob, flags=flags, **kw)
    return token.cpu().numpy(), logprob.cpu().double().numpy(), flags.cpu().numpy()


def check(z, u, near=0, **kw):
    token, logprob, flags = run(z, u, **kw)
    kw = {{"temperature": "T"}.get(k, k): v for k, v in kw.items()}
    zd, ud, skipped = z.cpu().double().numpy(), u.cpu().numpy(), 0
    for r in range(len(zd)):
        t, lp, margin = O.draw(zd[r], ud[r], **kw)
        assert flags[r] == (1 if t < 0 else 0)
        if margin < 1e-12:
            skipped += 1
            continue
        assert token[r] == t, (r, token[r], t, margin)
        assert np.isnan(logprob[r]) if t < 0 else abs(logprob[r] - lp) <= 2.0 ** -24 * abs(lp) + 1e-12, (r, logprob[r], lp)
    assert skipped <= near
    return token


WARPS = [dict(), dict(temperature=0.7, top_k=20, top_p=0.8), dict(top_p=0.95), dict(top_p=0.5, temperature=1.5), dict(top_k=1), dict(top_k=50),
         dict(min_p=0.1), dict(min_p=1.0), dict(top_p=0.9, min_p=0.05), dict(top_k=1000), dict(top_k=1500, top_p=0.9, min_p=0.001),
         dict(top_p=0.999, temperature=2.0), dict(top_k=300, min_p=1e-6), dict(temperature=0.05), dict(top_p=1e-6)]


@pytest.mark.parametrize("warp", WARPS, ids=str)
@pytest.mark.parametrize("V, dtype", [(1, F32), (7, BF16), (64, F32), (1000, BF16), (4099, F32), (32001, BF16), (50000, F32)])
def test_warps(V, dtype, warp):
    z, u = logits(12, V, dtype, V)
    check(z, u, **warp)


@pytest.mark.parametrize("warp", WARPS, ids=str)
@pytest.mark.parametrize("spread", [0.0, 0.02, 0.5])
def test_flat_rows(spread, warp):
    """Rows whose warps reach thousands of entries, and rows of one value (all of them tie)."""
    for dtype in (F32, BF16):
        z, u = logits(4, 20000, dtype, 3, spread)
        if spread == 0.0:
            z = torch.full_like(z, 1.5)
        check(z, u, **warp)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_headline_vocabulary(dtype):
    z, u = logits(6, 152064, dtype, 11)
    for warp in WARPS[:4] + WARPS[8:11]:
        check(z, u, **warp)


def test_edges_of_the_random_numbers():
    z, _ = logits(6, 3001, F32, 5)
    u = torch.tensor([0.0, 1.0 - 2.0 ** -53, 1.0, -0.5, 7.0, float("nan")], dtype=torch.float64, device="cuda")
    for warp in WARPS[:3]:
        token = check(z, u, near=6, **warp)
        assert (token[:5] >= 0).all() and token[5] == -1
        assert (token[:5] < 3001).all()


def test_every_token_at_its_share():
    """Random numbers on a fine grid draw each token as often as its probability says, to one."""
    p = np.array([0.5, 0.0, 0.25, 0.125, 0.125, 0.0])
    n = 4096
    with np.errstate(divide="ignore"):
        z = torch.from_numpy(np.log(p)).float().expand(n, 6).contiguous().cuda()
    u = (torch.arange(n, dtype=torch.float64) + 0.5).cuda() / n
    token, logprob, _ = run(z, u)
    assert (np.abs(np.bincount(token, minlength=6) - n * p) <= 1).all()
    assert np.allclose(logprob, np.log(p[token]), atol=1e-6)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_and_bad_rows(dtype):
    V = 9001
    z, u = logits(9, V, dtype, 8)
    low = torch.finfo(dtype).min
    z[0, :] = float("-inf")
    z[0, [5, 8999]] = 0.0
    z[1, 1:] = low                                        # the type's lowest value as a mask
    z[2, :] = float("-inf")
    z[3, :] = low
    z[4, 17] = float("nan")
    z[5, 17] = float("inf")
    z[6, 9000] = float("nan")
    z[7, :9000] = float("-inf")
    for warp in WARPS:
        token = check(z, u, **warp)
        assert (token[[2, 3, 4, 5, 6]] == -1).all() and token[1] == 0 and token[7] == 9000 and token[0] in (5, 8999)


def test_strides_streams_and_replays():
    z, u = logits(5, 5001, BF16, 9, pad=7)
    assert not z.is_contiguous()
    ref = check(z, u, top_p=0.9)
    token = torch.zeros(5, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    P.sv_sample(z, u, token, top_p=0.9, stream=s)
    s.synchronize()
    assert np.array_equal(token.cpu().numpy(), ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.sv_sample(z, u, token, top_p=0.9)
    for seed in range(4):
        z2, u2 = logits(5, 5001, BF16, 20 + seed, pad=7)
        z.copy_(z2)
        u.copy_(u2)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(token.cpu().numpy(), check(z, u, top_p=0.9))


def test_rows_beyond_32_bits():
    """4.4e9 elements: the last rows."""
    V, rows = 152064, 29000
    z = torch.full((rows, V), -1.0, dtype=BF16, device="cuda")
    want = torch.randint(0, V, (3,), generator=torch.Generator().manual_seed(1))
    for i in range(3):
        z[rows - 3 + i, want[i]] = 100.0
    u = torch.full((rows,), 0.5, dtype=torch.float64, device="cuda")
    token = torch.zeros(rows, dtype=torch.int32, device="cuda")
    P.sv_sample(z, u, token, top_k=5)
    assert np.array_equal(token[-3:].cpu().numpy(), want.numpy())


@pytest.mark.parametrize("V, dtype", [(170001, F32), (330001, BF16), (500009, F32)])
def test_vocabularies_that_share_maxima(V, dtype):
    """More vectors than there are maxima kept of them."""
    z, u = logits(3, V, dtype, 12)
    for warp in WARPS[:4] + WARPS[5:10]:
        check(z, u, **warp)


@pytest.mark.parametrize("K", [2048, 2049, 5000, 19999, 20000, 20001])
def test_many_entries_left(K):
    for dtype in (F32, BF16):
        z, u = logits(3, 20000, dtype, K)
        for warp in (dict(), dict(top_p=0.9), dict(top_p=0.7, min_p=1e-5, temperature=3.0)):
            check(z, u, top_k=K, **warp)


def test_no_rows():
    P.sv_sample(torch.empty((0, 8), device="cuda"), torch.empty(0, dtype=torch.float64, device="cuda"),
                torch.empty(0, dtype=torch.int32, device="cuda"))
