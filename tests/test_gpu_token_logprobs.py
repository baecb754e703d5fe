"""sv_token_logprobs and sv_token_logprobs_grad against the fp64 definitions.

Tolerances.  A term 2^y of a row's sum has the error of its exponent's rounding, |y| 2^-24 ln 2 with |y| <= 24 for
the terms that carry a sum, and that of v_exp_f32, 1.2e-7: below 1.2e-6, and so is the sum's.  The temperature is
off by 6e-8 at most, to first order about the maximum only: 12 nats of distance to it are 7e-7.  Hence 2e-6 for a
normaliser or log-probability, plus the result's rounding.  The entropy's error is the terms' (1.2e-6) times the
spread of -log p (4 nats at most here), plus the rounding of 2^y y: 6e-6.  A gradient entry has the errors of its
probability and of the sum, and of log p + H where there is an entropy term; bfloat16 results are the one rounding of such a number."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
from oracle import operators_oracle as O
from paper_2509_24328_amd import binding as Bd

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
NAN = float("nan")


def bits(t):
    t = t.detach().cpu().contiguous()
    return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == BF16 else t.numpy()


def logits(N, V, dtype, seed, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    z = 2.5 * torch.randn((N, V), generator=g)
    if kind == "few":                                   # many equal logits
        z = torch.randint(-3, 4, (N, V), generator=g).float()
    elif kind == "flat":
        z = torch.full((N, V), 0.75)
    elif kind == "rising":                              # every vector holds a new maximum
        z = torch.arange(V).float().expand(N, V) * (8.0 / V) + 1e-3 * z
    elif kind == "masked":                              # a few tokens allowed, the others at -inf or at the lowest number
        low = -float("inf") if seed % 2 else torch.finfo(dtype).min
        keep = torch.rand((N, V), generator=g) < 6.0 / V
        keep[:, V // 2] = True
        z = torch.where(keep, z, torch.tensor(low))
    elif kind == "peaks":                               # the largest entries lie one workgroup's stride apart
        z[:, 5::8192] += 30.0
    elif kind == "shifted":
        z = z + 300.0
    return z.to(dtype)


def score(z, tokens, n_top=0, T=1.0, offsets=None, shape=None):
    """All outputs, over poisoned buffers."""
    shape = tuple(tokens.shape) if shape is None else shape
    f = lambda *s: torch.full(shape + s, 12345.0, device="cuda")
    i = lambda *s: torch.full(shape + s, -777, dtype=torch.int32, device="cuda")
    out = dict(logprob=f(), lse=f(), entropy=f(), rank=i(), flags=i())
    if n_top:
        out.update(top_token=i(n_top), top_logprob=f(n_top))
    P.sv_token_logprobs(z, tokens, out["logprob"], out["lse"], out["entropy"], out["rank"], out.get("top_token"),
                        out.get("top_logprob"), out["flags"], T, offsets)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in out.items()}


def same(got, ref, n_top):
    for k in ("rank", "flags") + (("top_token",) if n_top else ()):
        assert np.array_equal(got[k].reshape(ref[k].shape), ref[k]), k
    for k, tol in (("logprob", 2e-6), ("lse", 2e-6), ("entropy", 6e-6)) + ((("top_logprob", 2e-6),) if n_top else ()):
        a, b = got[k].reshape(ref[k].shape).astype(np.float64), ref[k]
        fin = np.isfinite(b)
        assert np.array_equal(a[~fin], b[~fin], equal_nan=True), k
        assert (np.abs(a[fin] - b[fin]) <= tol + 1.3e-7 * np.abs(b[fin])).all(), (k, np.abs(a[fin] - b[fin]).max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 33, 509, 4096, 8193, 32001])
@pytest.mark.parametrize("n_top", [0, 1, 5, 32])
def test_sizes(dtype, V, n_top):
    N = 5
    z = logits(N, V, dtype, V + n_top)
    tok = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(V), dtype=torch.int32)
    tok[1] = -1
    got = score(z.cuda(), tok.cuda(), n_top)
    same(got, O.token_logprobs(bits(z), tok.numpy(), 1.0, n_top), n_top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["few", "flat", "rising", "masked", "peaks", "shifted"])
@pytest.mark.parametrize("V", [1000, 32000, 70001])
def test_distributions(dtype, kind, V):
    N, n_top = 4, 20
    for seed in (10, 11):
        z = logits(N, V, dtype, seed, kind)
        tok = torch.tensor([0, V - 1, V // 2, V // 3], dtype=torch.int32)
        got = score(z.cuda(), tok.cuda(), n_top, 0.75 if seed == 11 else 1.0)
        same(got, O.token_logprobs(bits(z), tok.numpy(), 0.75 if seed == 11 else 1.0, n_top), n_top)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [1e-3, 0.3, 1.0, 17.0, 1e3])
def test_temperatures(dtype, T):
    """The distance to the maximum is what a temperature's error is multiplied by: y up to 2^14 at T = 1e-3."""
    z = logits(3, 5000, dtype, 7)
    tok = z.float().argmax(-1).to(torch.int32)
    T = float(np.float32(T))
    same(score(z.cuda(), tok.cuda(), 3, T), O.token_logprobs(bits(z), tok.numpy(), T, 3), 3)


def test_zeros_of_both_signs_are_equal():
    z = torch.full((1, 40), -1.0)
    z[0, 3::5] = 0.0
    z[0, 1::7] = -0.0
    for dtype in (F32, BF16):
        tok = torch.tensor([22], dtype=torch.int32)
        same(score(z.to(dtype).cuda(), tok.cuda(), 14), O.token_logprobs(bits(z.to(dtype)), tok.numpy(), 1.0, 14), 14)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_conditions(dtype):
    """NaN, +inf, nothing left, tokens out of range, masked tokens, one entry left."""
    V = 600
    z = logits(9, V, dtype, 3)
    z[0, 555] = NAN
    z[1, 0] = float("inf")
    z[2] = -float("inf")
    z[3] = torch.finfo(dtype).min
    z[4, 17] = -float("inf")
    z[7] = -float("inf")
    z[7, V - 1] = -2.0
    tok = torch.tensor([1, 1, 1, 1, 17, V, -2, 3, -1], dtype=torch.int32)
    ref = O.token_logprobs(bits(z), tok.numpy(), 1.0, 4)
    assert ref["flags"].tolist() == [1, 1, 1, 1, 0, 16, 16, 0, 0]
    same(score(z.cuda(), tok.cuda(), 4), ref, 4)
    # without tokens every row is swept
    out = {k: torch.empty(9, device="cuda") for k in ("lse", "entropy")}
    top, val = torch.empty((9, 4), dtype=torch.int32, device="cuda"), torch.empty((9, 4), device="cuda")
    P.sv_token_logprobs(z.cuda(), None, None, out["lse"], out["entropy"], None, top, val)
    ref = O.token_logprobs(bits(z), None, 1.0, 4)
    assert np.array_equal(top.cpu().numpy(), ref["top_token"])
    assert np.allclose(out["lse"].cpu().numpy(), ref["lse"], rtol=1e-6, atol=2e-6, equal_nan=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_rows_padding_and_strides(dtype):
    B, Pn, V, n_top = 5, 4, 777, 3
    count = torch.tensor([4, 0, 1, 3, 2])
    offs = torch.cat([torch.zeros(1, dtype=torch.long), count.cumsum(0)]).to(torch.int32)
    R = int(offs[-1])
    wide = torch.full((R, V + 19), 50.0, dtype=dtype)
    wide[:, :V] = logits(R, V, dtype, 5)
    tok = torch.randint(0, V, (B, Pn), dtype=torch.int32)
    tok[0, 2] = -1
    z = wide.cuda()[:, :V]
    got = score(z, tok.cuda(), n_top, offsets=offs.cuda())
    flat = np.full(B * Pn, -1)
    rows = np.zeros((B * Pn, V), bits(wide).dtype)
    for b in range(B):
        for i in range(int(count[b])):
            flat[b * Pn + i] = int(tok[b, i])
            rows[b * Pn + i] = bits(wide[:, :V])[int(offs[b]) + i]
    ref = O.token_logprobs(rows, flat, 1.0, n_top)
    same(got, ref, n_top)
    # rows that the offsets place outside z are bad, and never read
    far = offs.clone()
    far[3:] += 100
    got = score(z, tok.cuda(), n_top, offsets=far.cuda())
    assert (got["flags"][4, :2] == 1).all() and np.isnan(got["lse"][4, :2]).all() and (got["top_token"][4] == -1).all()
    far = offs - 2
    got = score(z, tok.cuda(), n_top, offsets=far.cuda())
    assert got["flags"][0, 0] == 1 and got["flags"][0, 1] == 1 and got["flags"][0, 3] == 0
    # dense positions in wider rows, starting on any element
    store = torch.zeros(B * Pn * (V + 3) + 1, dtype=dtype)
    zd = logits(B * Pn, V, dtype, 6)
    view = store[1:].view(B, Pn, V + 3)
    view[..., :V] = zd.view(B, Pn, V)
    dev = store.cuda()[1:].view(B, Pn, V + 3)[..., :V]
    same(score(dev, tok.cuda(), n_top), O.token_logprobs(bits(zd), tok.numpy().ravel(), 1.0, n_top), n_top)


def test_rows_beyond_32_bits():
    V, N = 128256, 34000                                # 4.4e9 elements
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    z = torch.empty((N, V), dtype=BF16, device="cuda")
    tok = torch.full((N,), -1, dtype=torch.int32)
    some = [0, 16744, 33487, N - 1]
    part = logits(len(some), V, BF16, 1)
    for j, r in enumerate(some):
        z[r] = part[j].cuda()
        tok[r] = 1000 * j
    got = score(z, tok.cuda(), 2)
    ref = O.token_logprobs(bits(part), tok[some].numpy(), 1.0, 2)
    same({k: v[some] for k, v in got.items()}, ref, 2)
    rest = np.setdiff1d(np.arange(N), some)
    assert not got["lse"][rest].any() and (got["top_token"][rest] == -1).all()
    g = torch.ones(N, device="cuda")
    P.sv_token_logprobs_grad(z, tok.cuda(), g, z)       # in place
    for j, r in enumerate(some):
        ref = O.token_logprobs_grad(bits(part[j:j + 1]), [1000 * j], [1.0])["dz"][0]
        assert np.abs(O.values(bits(z[r])) - ref).max() <= 2.0 ** -8
    assert not z[1].any() and not z[N - 2].any()


# ---------------------------------------------------------------------------
# gradient
# ---------------------------------------------------------------------------
def check_grad(z, tok, g, h, T, got):
    ref = O.token_logprobs_grad(bits(z), tok.numpy(), g.double().numpy(), None if h is None else h.double().numpy(), T)
    N, V = z.shape
    dz = O.values(bits(got["dz"]))
    assert np.array_equal(got["flags"].cpu().numpy(), ref["flags"])
    for k, tol in (("logprob", 2e-6), ("entropy", 6e-6)):
        a = got[k].cpu().numpy().astype(np.float64)
        assert np.allclose(a, ref[k], rtol=1.3e-7, atol=tol, equal_nan=True), k
    for r in range(N):
        b = ref["dz"][r]
        if np.isnan(b).any():
            assert np.isnan(dz[r]).all()
            continue
        p = ref["p"][r]
        with np.errstate(divide="ignore", invalid="ignore"):
            lp = np.where(p > 0, np.log(p), 0.0)
        hh = 0.0 if h is None else abs(float(h[r]))
        gg = abs(float(g[r]))
        of_p = 2.5e-6 + 1.3e-7 * np.abs(lp) / np.log(2)
        tol = p / T * (gg * of_p + hh * ((np.abs(lp) + ref["entropy"][r]) * of_p + 7e-6)) + 2.4e-7 * np.abs(b) + 1e-36
        t = int(tok[r])
        if 0 <= t < V:
            tol[t] += 2.4e-7 * gg / T
        fine = O.within(dz[r], b, tol, z.dtype == BF16)
        assert fine.all(), (r, int(fine.argmin()), float(dz[r][fine.argmin()]), float(b[fine.argmin()]))


def run_grad(z, tok, g, h, T=1.0, dz=None):
    N = z.shape[0]
    out = dict(logprob=torch.full((N,), 9.0, device="cuda"), entropy=torch.full((N,), 9.0, device="cuda"),
               flags=torch.full((N,), 9, dtype=torch.int32, device="cuda"),
               dz=torch.full_like(z, 9.0) if dz is None else dz)
    P.sv_token_logprobs_grad(z, tok.cuda(), g.cuda(), out["dz"], None if h is None else h.cuda(), out["logprob"],
                             out["entropy"], out["flags"], T)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1, 3, 8, 100, 4099, 32768, 40007, 152064])
@pytest.mark.parametrize("entropy", [False, True])
def test_gradient(dtype, V, entropy):
    N = 4
    z = logits(N, V, dtype, V)
    gen = torch.Generator().manual_seed(V)
    tok = torch.randint(0, V, (N,), generator=gen, dtype=torch.int32)
    tok[2] = -1
    g = torch.randn(N, generator=gen)
    h = torch.randn(N, generator=gen) if entropy else None
    T = 0.75 if V % 2 else 1.0
    check_grad(z, tok, g, h, T, run_grad(z.cuda(), tok, g, h, T))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["few", "flat", "rising", "masked", "peaks", "shifted"])
def test_gradient_of_distributions(dtype, kind):
    V, N = 20011, 3
    for seed in (20, 21):
        z = logits(N, V, dtype, seed, kind)
        tok = torch.tensor([V // 2, 0, V - 1], dtype=torch.int32)
        g, h = torch.tensor([1.0, -0.5, 3.0]), torch.tensor([0.1, 0.0, -2.0])
        check_grad(z, tok, g, h, 1.0, run_grad(z.cuda(), tok, g, h))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_conditions_in_place_and_strides(dtype):
    V, N = 501, 8
    z = logits(N, V, dtype, 3)
    z[0, 500] = NAN
    z[1, 0] = float("inf")
    z[2] = -float("inf")
    z[3, 17] = -float("inf")
    tok = torch.tensor([1, 1, 1, 17, V, -2, -1, 3], dtype=torch.int32)
    g, h = torch.randn(N, generator=torch.Generator().manual_seed(1)), torch.full((N,), 0.25)
    check_grad(z, tok, g, h, 1.0, run_grad(z.cuda(), tok, g, h))
    check_grad(z, tok, g, None, 1.0, run_grad(z.cuda(), tok, g, None))
    zz = z.cuda()
    check_grad(z, tok, g, h, 1.0, run_grad(zz, tok, g, h, dz=zz))
    # wider rows on both sides: the columns past V stay
    a, b = torch.full((N, V + 6), 4.0, dtype=dtype), torch.full((N, V + 11), 5.0, dtype=dtype)
    a[:, :V] = z
    a, b = a.cuda(), b.cuda()
    check_grad(z, tok, g, h, 1.0, run_grad(a[:, :V], tok, g, h, dz=b[:, :V]))
    assert (b[:, V:] == 5.0).all()


def test_gradient_against_differences():
    """Central differences of the call's own log-probability and entropy, in float32 outputs: with steps of 1/8 the
    rounding of the sums is 8e-6 / 0.25 and the truncation step^2 / 6 times a third derivative below 1."""
    V, N = 12, 2
    z = torch.round(logits(N, V, F32, 4) * 64) / 64
    tok = torch.tensor([3, 11], dtype=torch.int32)
    g, h = torch.tensor([1.0, -0.7]), torch.tensor([0.3, 0.9])
    dz = run_grad(z.cuda(), tok, g, h)["dz"].cpu().numpy()
    step = 0.125

    def value(zz):
        o = score(zz.cuda(), tok.cuda())
        return o["logprob"].astype(np.float64) * g.numpy() + o["entropy"].astype(np.float64) * h.numpy()

    for v in range(V):
        up, down = z.clone(), z.clone()
        up[:, v] += step
        down[:, v] -= step
        est = (value(up) - value(down)) / (2 * step)
        assert (np.abs(est - dz[:, v]) <= 4e-5 + step ** 2 / 6).all(), v


def test_other_streams_and_graphs():
    V, N, n_top = 32000, 6, 5
    z = logits(N, V, BF16, 8).cuda()
    tok = torch.arange(N, dtype=torch.int32).cuda()
    g = torch.ones(N, device="cuda")
    want = score(z, tok, n_top)
    out = dict(logprob=torch.empty(N, device="cuda"), top=torch.empty((N, n_top), dtype=torch.int32, device="cuda"),
               val=torch.empty((N, n_top), device="cuda"), dz=torch.empty_like(z))
    call = lambda s=None: (P.sv_token_logprobs(z, tok, out["logprob"], top_token=out["top"], top_logprob=out["val"], stream=s),
                           P.sv_token_logprobs_grad(z, tok, g, out["dz"], stream=s))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(side)
    side.synchronize()
    assert np.array_equal(out["logprob"].cpu().numpy(), want["logprob"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        z.copy_(logits(N, V, BF16, 30 + k).cuda())
        for t in out.values():
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        want = score(z, tok, n_top)
        assert np.array_equal(out["logprob"].cpu().numpy(), want["logprob"])
        assert np.array_equal(out["top"].cpu().numpy(), want["top_token"])
        dz = run_grad(z, tok.cpu(), g.cpu(), None)["dz"]
        assert torch.equal(dz, out["dz"])


def test_refusals():
    z = torch.zeros((2, 8), device="cuda")
    tok = torch.zeros(2, dtype=torch.int32, device="cuda")
    f = torch.zeros(2, device="cuda")
    cases = [
        (Bd.SV_ERR_DTYPE, lambda: P.sv_token_logprobs(z.half(), tok, f)),
        (Bd.SV_ERR_DTYPE, lambda: P.sv_token_logprobs(z, tok.long(), f)),
        (Bd.SV_ERR_DTYPE, lambda: P.sv_token_logprobs(z, tok, f.double())),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_token_logprobs(z, tok, f, temperature=0.0)),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_token_logprobs(z, tok, f, temperature=NAN)),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_token_logprobs(z, tok[:1], f)),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_token_logprobs(z, tok, f[:1])),
        (Bd.SV_ERR_NULL, lambda: P.sv_token_logprobs(z, None, f)),
        (Bd.SV_ERR_NULL, lambda: P.sv_token_logprobs(z, tok, f, top_token=torch.zeros((2, 3), dtype=torch.int32, device="cuda"))),
        (Bd.SV_ERR_TOO_LARGE, lambda: P.sv_token_logprobs(z, tok, f, top_token=torch.zeros((2, 33), dtype=torch.int32, device="cuda"),
                                                          top_logprob=torch.zeros((2, 33), device="cuda"))),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_token_logprobs_grad(z, tok, f, z[:, :7])),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_token_logprobs_grad(z, tok, f, z.bfloat16())),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_token_logprobs_grad(z, tok, f, z.clone(), temperature=2e3)),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_token_logprobs_grad(z, tok, f[:1], z.clone())),
    ]
    for code, call in cases:
        with pytest.raises(P.SvError) as e:
            call()
        assert e.value.status == code
    with pytest.raises(ValueError):
        P.sv_token_logprobs(z.cpu(), tok, f)
    with pytest.raises(ValueError):
        P.sv_token_logprobs(torch.zeros((8, 2), device="cuda").t(), tok, f)
    P.sv_token_logprobs(z[:0], tok[:0], f[:0])
    P.sv_token_logprobs_grad(z[:0], tok[:0], f[:0], z[:0].clone())
