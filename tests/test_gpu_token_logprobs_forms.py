"""The scoring calls and their gradient at the sizes that choose another kernel: rows in the registers of 1024 lanes and past
them, many short rows, rows that several workgroups share (with all that can be wrong with a row), and logits past the
last-level cache.  Most positions of the large calls have no token, and are checked to be blank.  Tolerances: those derived in
test_gpu_token_logprobs."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
from oracle import operators_oracle as O
from test_gpu_token_alternatives import check as check_alternatives
from test_gpu_token_logprobs import bits, check_grad, logits, run_grad, same, score

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def scattered(N, V, dtype, seed, rows, token=None):
    """z [N, V] on the GPU, tokens (-1 but at `rows`), those rows' logits and tokens.  Rows without a token are NaN: never read."""
    part = logits(len(rows), V, dtype, seed)
    z = torch.full((N, V), float("nan"), dtype=dtype, device="cuda")
    z[rows] = part.cuda()
    some = torch.randint(0, V, (len(rows),), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    some[0], some[-1] = V - 1, 0
    tok = torch.full((N,), -1, dtype=torch.int32)
    tok[rows] = some if token is None else token
    return z, tok, part, tok[rows]


def blank(got, rows, n_top=0):
    rest = np.setdiff1d(np.arange(len(got["logprob"])), rows)
    for k in ("logprob", "lse", "entropy", "rank", "flags"):
        assert not got[k][rest].any(), k
    if n_top:
        assert (got["top_token"][rest] == -1).all() and (got["top_logprob"][rest] == -np.inf).all()


# ---------------------------------------------------------------------------
# gradient: one workgroup to a row (more than 96 rows)
# ---------------------------------------------------------------------------
# vectors of a row: up to 2048, 4096 and 8192 have 8, 8 and 12 registers of 256, 512 and 512 lanes (6144 vectors of the last), longer ones 19
# of 1024 (19456): below, at and above each of these, with and without entries past the last whole vector
@pytest.mark.parametrize("vectors", [2048, 2049, 4096, 4097, 6144, 6145, 8192, 8193, 19008, 19456, 19457, 22501])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("entropy, in_place, over", [(False, False, 0), (True, False, -1), (True, True, 0), (False, True, 1)])
def test_gradient_by_one_workgroup(vectors, dtype, entropy, in_place, over):
    N, V = 193, vectors * (4 if dtype == F32 else 8) + over
    rows = [0, 77, N - 1]
    z, tok, part, some = scattered(N, V, dtype, vectors, rows)
    gen = torch.Generator().manual_seed(vectors)
    g = torch.randn(N, generator=gen)
    h = torch.randn(N, generator=gen) if entropy else None
    T = 0.75 if over else 1.0
    out = run_grad(z, tok, g, h, T, dz=z if in_place else None)
    rest = torch.from_numpy(np.setdiff1d(np.arange(N), rows)).cuda()
    assert not out["dz"][rest].any() and not out["logprob"][rest].any() and not out["entropy"][rest].any()
    check_grad(part, some, g[rows], None if h is None else h[rows], T, {k: v[rows] for k, v in out.items()})


# ---------------------------------------------------------------------------
# rows that several workgroups share: from ten rounds of 1024 vectors on, up to 96 rows (gradient) and 682
# ---------------------------------------------------------------------------
def conditions(N, V, dtype, seed):
    """Rows with NaN, +inf, nothing left, the lowest number alone, a masked token, one entry left, and what is wrong in one part only."""
    z = logits(N, V, dtype, seed)
    z[0, V - 1] = float("nan")
    z[1, 0] = float("inf")
    z[2] = -float("inf")
    z[3] = torch.finfo(dtype).min
    z[4, 17] = -float("inf")
    z[5] = -float("inf")
    z[5, V - 1] = -2.0
    z[6, :V // 2] = -float("inf")
    z[7, V // 3:] = torch.finfo(dtype).min
    tok = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    tok[:12] = torch.tensor([1, 1, 1, 1, 17, V - 1, V - 1, V - 1, V, -2, -1, V - 2])
    return z, tok


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rounds", [10, 19])             # a key of every lane of the sweep, and one of four
@pytest.mark.parametrize("T", [1.0, 0.75])
def test_conditions_of_shared_rows(dtype, rounds, T):
    N, V, n_top = 13, (1024 * rounds - 300) * (4 if dtype == F32 else 8) + 3, 7
    tag = P.SV_F32 if dtype == F32 else P.SV_BF16
    assert P.sv_token_logprobs_workspace_bytes(N, V, tag, n_top) > 0
    z, tok = conditions(N, V, dtype, rounds)
    ref = O.token_logprobs(bits(z), tok.numpy(), T, n_top)
    assert ref["flags"].tolist() == [1, 1, 1, 1, 0, 0, 0, 0, 16, 16, 0, 0, 0]
    same(score(z.cuda(), tok.cuda(), n_top, T), ref, n_top)
    same(score(z.cuda(), tok.cuda(), 0, T), {k: v for k, v in ref.items() if "top" not in k}, 0)
    # wider rows that start on any element
    store = torch.zeros(N * (V + 3) + 1, dtype=dtype, device="cuda")
    view = store[1:].view(N, V + 3)
    view[:, :V] = z.cuda()
    view[:, V:] = 60.0
    same(score(view[:, :V], tok.cuda(), n_top, T), ref, n_top)
    # the gradient, beside and in place of the logits, with their padding
    gen = torch.Generator().manual_seed(1)
    g, h = torch.randn(N, generator=gen), torch.randn(N, generator=gen)
    check_grad(z, tok, g, h, T, run_grad(z.cuda(), tok, g, h, T))
    check_grad(z, tok, g, None, T, run_grad(view[:, :V], tok, g, None, T, dz=view[:, :V]))
    assert (view[:, V:] == 60.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_shared_rows(dtype):
    B, Pn, n_top, V = 4, 3, 5, 85001
    count = torch.tensor([3, 0, 1, 2])
    offs = torch.cat([torch.zeros(1, dtype=torch.long), count.cumsum(0)]).to(torch.int32)
    R = int(offs[-1])
    wide = torch.full((R, V + 5), 50.0, dtype=dtype)
    wide[:, :V] = logits(R, V, dtype, 5)
    wide[2, 5] = float("nan")
    tok = torch.randint(0, V, (B, Pn), generator=torch.Generator().manual_seed(4), dtype=torch.int32)
    tok[0, 1], tok[2, 0] = -1, V
    assert P.sv_token_logprobs_workspace_bytes(B * Pn, V, P.SV_BF16, n_top) > 0
    z = wide.cuda()[:, :V]
    for move in (0, -2, 3):                              # rows that the offsets place outside z are bad, and never read
        got = score(z, tok.cuda(), n_top, offsets=(offs + move).cuda())
        flat, rows = np.full(B * Pn, -1), np.zeros((B * Pn, V), bits(wide).dtype)
        out_of_z = np.zeros(B * Pn, bool)
        for b in range(B):
            for i in range(int(count[b])):
                r = int(offs[b]) + i + move
                if int(tok[b, i]) == -1:
                    continue
                out_of_z[b * Pn + i] = not 0 <= r < R
                flat[b * Pn + i] = -1 if out_of_z[b * Pn + i] else int(tok[b, i])
                rows[b * Pn + i] = bits(wide[:, :V])[min(max(r, 0), R - 1)]
        ref = O.token_logprobs(rows, flat, 1.0, n_top)
        for k in ("logprob", "lse", "entropy", "top_logprob"):
            ref[k][out_of_z] = np.nan
        ref["flags"][out_of_z] = 1
        assert out_of_z.sum() == (0 if move == 0 else 1 if move == -2 else 3)
        same(got, ref, n_top)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_longest_row(dtype):
    """2^24 entries: 64 parts."""
    V = 1 << 24
    z = logits(1, V, dtype, 12)
    check_alternatives(z, 20)
    tok = torch.tensor([V - 1], dtype=torch.int32)
    g, h = torch.tensor([1.5]), torch.tensor([-0.5])
    check_grad(z, tok, g, h, 1.0, run_grad(z.cuda(), tok, g, h))


# ---------------------------------------------------------------------------
# scoring: many short rows, and logits past the last-level cache
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_top", [0, 1, 20, 32])
@pytest.mark.parametrize("V", [1, 300, 2003])
def test_many_short_rows(dtype, n_top, V):
    """1024 rows of at most 4096 vectors have workgroups of 256 lanes."""
    N = 1030
    z = logits(N, V, dtype, V + n_top, "few" if n_top == 20 else "normal")
    tok = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(V), dtype=torch.int32)
    tok[5], tok[6], tok[N - 2] = -1, V, -3
    z[8, V // 2] = float("nan")
    z[9] = -float("inf")
    same(score(z.cuda(), tok.cuda(), n_top), O.token_logprobs(bits(z), tok.numpy(), 1.0, n_top), n_top)


@pytest.mark.parametrize("dtype, N, V", [
    (F32, 1040, 16384), (F32, 1040, 16385), (BF16, 1040, 32768), (BF16, 1040, 32769),      # at 4096 vectors and above
    (BF16, 40000, 2003), (F32, 20000, 2003),             # 256 lanes, past the cache
    (F32, 1100, 32001), (BF16, 2200, 32001),             # 512 lanes, past the cache
    (F32, 300, 152064), (BF16, 600, 152064),             # shared rows, past the cache
    (F32, 683, 60001), (BF16, 683, 100003)])             # one row more than are shared
@pytest.mark.parametrize("n_top", [0, 20])
def test_large_calls(dtype, N, V, n_top):
    rows = [0, N // 3, N // 2, N - 1]
    z, tok, part, some = scattered(N, V, dtype, V, rows)
    got = score(z, tok.cuda(), n_top)
    same({k: v[rows] for k, v in got.items()}, O.token_logprobs(bits(part), some.numpy(), 1.0, n_top), n_top)
    blank(got, rows, n_top)


# ---------------------------------------------------------------------------
# scratch that the binding takes
# ---------------------------------------------------------------------------
def test_scratch_on_other_streams_and_in_graphs():
    """Shared rows: scratch is torch's, on the stream of the call; calls that follow may be handed the same."""
    V, N, n_top = 152064, 6, 5
    assert P.sv_token_logprobs_workspace_bytes(N, V, P.SV_BF16, n_top) > 0
    z = logits(N, V, BF16, 8).cuda()
    tok = torch.arange(N, dtype=torch.int32).cuda()
    g = torch.ones(N, device="cuda")
    out = dict(logprob=torch.empty(N, device="cuda"), top=torch.empty((N, n_top), dtype=torch.int32, device="cuda"),
               val=torch.empty((N, n_top), device="cuda"), dz=torch.empty_like(z))

    def call(s=None):
        P.sv_token_logprobs(z, tok, out["logprob"], top_token=out["top"], top_logprob=out["val"], stream=s)
        P.sv_token_logprobs_grad(z, tok, g, out["dz"], stream=s)

    def fine():
        want = score(z, tok, n_top)
        assert np.array_equal(out["logprob"].cpu().numpy(), want["logprob"])
        assert np.array_equal(out["top"].cpu().numpy(), want["top_token"])
        assert np.array_equal(out["val"].cpu().numpy(), want["top_logprob"])
        assert torch.equal(out["dz"], run_grad(z, tok.cpu(), g.cpu(), None)["dz"])

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        call(side)
        with torch.cuda.stream(side):                    # what a call's scratch was is anyone's on that stream after it
            torch.full((1 << 20,), float("nan"), device="cuda")
    call(side)
    side.synchronize()
    fine()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        z.copy_(logits(N, V, BF16, 30 + k).cuda())
        for t in out.values():
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        fine()
