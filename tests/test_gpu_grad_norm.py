"""sv_grad_norm and sv_clip_grad_norm against the fp64 definitions.  The squares and their sum are float64, so the
norm has the rounding of its float32 result, 6e-8; the factor has that of the norm and its own, a clipped gradient
one more: 2e-7, before the one rounding to bfloat16."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
from oracle import operators_oracle as O
from paper_2509_24328_amd import binding as Bd

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def bits(t):
    t = t.detach().cpu().contiguous()
    return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == BF16 else t.numpy()


def make(sizes, kinds, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(size * torch.randn(s, generator=g)).to(k).cuda() for s, k in zip(sizes, kinds)]


def workspace(n):
    return torch.empty(P.sv_grad_norm_workspace_bytes(n), dtype=torch.uint8, device="cuda").fill_(255)


def check(grads, max_norm, out=None, out_kinds=None):
    n = len(grads)
    ref = O.grad_norm([bits(g) for g in grads])
    norm, flag = torch.full((1,), 9.0, device="cuda"), torch.full((1,), 9, dtype=torch.int32, device="cuda")
    P.sv_grad_norm(grads, norm, flag, workspace(n))
    assert abs(float(norm) - ref) <= 1.3e-7 * ref and int(flag) == 0
    before = [bits(g).copy() for g in grads]
    norm.fill_(9.0)
    P.sv_clip_grad_norm(grads, max_norm, norm, out, flag, workspace(n))
    assert abs(float(norm) - ref) <= 1.3e-7 * ref and int(flag) == 0
    by = O.clip_factor(ref, max_norm)
    for b, g, o in zip(before, grads, out if out is not None else grads):
        if out is not None:
            assert np.array_equal(bits(g), b)
        want = O.values(b) * by
        got = O.values(bits(o)).reshape(want.shape)
        assert O.within(got, want, 2e-7 * np.abs(want) + 1e-38, o.dtype == BF16).all()


SIZES = [1, 7, 8, 9, 1000, 16383, 16384, 16385, 100003]


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("max_norm", [0.5, 1e6, float("inf")])
def test_sizes(kind, max_norm):
    check(make(SIZES, [kind] * len(SIZES), 1), max_norm)
    for s in SIZES:
        check(make([s], [kind], s), max_norm)


@pytest.mark.parametrize("n", [1, 2, 119, 120, 121, 250, 400])
def test_many_tensors_of_both_types(n):
    """Also more tensors than one launch takes, and empty ones among them."""
    sizes = [(37 * i * i) % 5000 for i in range(n)]
    sizes[0] = 3
    kinds = [F32 if i % 3 == 0 else BF16 for i in range(n)]
    grads = make(sizes, kinds, n)
    out = [torch.full((s,), 5.0, dtype=F32 if i % 2 else BF16, device="cuda") for i, s in enumerate(sizes)]
    check(grads, 3.0, out)
    check(grads, 1e9, out)
    check(grads, 3.0)


def test_views_that_start_on_any_element():
    """Tensors and results are slices of one buffer, one after the other; what lies between stays."""
    sizes = [5, 17, 4099, 20001, 3]
    for kind in (F32, BF16):
        buf, to = torch.randn(30000, device="cuda").to(kind), torch.full((30000,), 8.0, dtype=kind, device="cuda")
        grads, out, at = [], [], 1
        for s in sizes:
            grads.append(buf[at:at + s])
            out.append(to[at:at + s])
            at += s + 2
        check(grads, 1.0, out)
        keep = torch.ones(30000, dtype=torch.bool)
        at = 1
        for s in sizes:
            keep[at:at + s] = False
            at += s + 2
        assert (to.cpu()[keep] == 8.0).all()


def test_many_granules():
    g = make([40_000_003, 11], [BF16, F32], 3, 1e-3)
    check(g, 1.0, [torch.empty_like(t) for t in g])


def test_large_and_small_numbers():
    """Squares that float32 does not hold."""
    check(make([1000, 30], [F32, F32], 4, 1e25), 1.0)
    check(make([1000, 30], [F32, BF16], 5, 1e-25), 1e-26)
    z = [torch.zeros(100, device="cuda")]
    check(z, 1.0)
    norm = torch.full((1,), 9.0, device="cuda")
    P.sv_grad_norm([], norm, ws=workspace(0))
    assert float(norm) == 0.0
    P.sv_clip_grad_norm([torch.empty(0, device="cuda")], 1.0, norm.fill_(9.0), ws=workspace(1))
    assert float(norm) == 0.0


@pytest.mark.parametrize("x", [float("nan"), float("inf"), -float("inf")])
def test_norm_that_is_not_finite(x):
    for kind in (F32, BF16):
        grads = make([100, 20000], [kind, F32], 6)
        grads[1][19999] = x
        before = [bits(g).copy() for g in grads]
        norm, flag = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        P.sv_clip_grad_norm(grads, 1.0, norm, None, flag, workspace(2))
        assert int(flag) == Bd.FLAG_NONFINITE and not np.isfinite(float(norm))
        assert all(np.array_equal(bits(g), b, equal_nan=b.dtype != np.uint16) for g, b in zip(grads, before))
        out = [torch.zeros_like(g) for g in grads]
        P.sv_clip_grad_norm(grads, 1.0, norm, out, flag, workspace(2))
        assert all(np.array_equal(bits(o), b, equal_nan=b.dtype != np.uint16) for o, b in zip(out, before))


def test_beyond_32_bits():
    n = (1 << 32) + 12345
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[0], g[1 << 31], g[n - 1] = 2.0, 3.0, 6.0
    norm = torch.zeros(1, device="cuda")
    P.sv_clip_grad_norm([g], 3.5, norm, ws=workspace(1))
    assert float(norm) == 7.0
    assert [float(g[0]), float(g[1 << 31]), float(g[n - 1])] == [1.0, 1.5, 3.0]


def test_the_same_bits_and_graphs():
    grads = make(SIZES * 20, [BF16] * (20 * len(SIZES)), 7)
    out = [torch.empty_like(g) for g in grads]
    norm, ws = torch.zeros(1, device="cuda"), workspace(len(grads))
    call = lambda s=None: P.sv_clip_grad_norm(grads, 10.0, norm, out, None, ws, s)
    call()
    want = float(norm)
    for _ in range(3):
        call()
        assert float(norm) == want
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(side)
    side.synchronize()
    assert float(norm) == want
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        for g, h in zip(grads, make(SIZES * 20, [BF16] * (20 * len(SIZES)), 70 + k)):
            g.copy_(h)
        call()
        want, kept = float(norm), [o.clone() for o in out]
        norm.zero_()
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert float(norm) == want and all(torch.equal(a, b) for a, b in zip(kept, out))


def test_refusals():
    g = [torch.zeros(8, device="cuda")]
    norm, ws = torch.zeros(1, device="cuda"), workspace(1)
    cases = [
        (Bd.SV_ERR_DTYPE, lambda: P.sv_grad_norm([g[0].half()], norm, ws=ws)),
        (Bd.SV_ERR_DTYPE, lambda: P.sv_grad_norm(g, norm.double(), ws=ws)),
        (Bd.SV_ERR_WORKSPACE, lambda: P.sv_grad_norm(g, norm)),
        (Bd.SV_ERR_WORKSPACE, lambda: P.sv_grad_norm(g, norm, ws=ws[:256])),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_clip_grad_norm(g, 0.0, norm, ws=ws)),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_clip_grad_norm(g, float("nan"), norm, ws=ws)),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_clip_grad_norm(g, 1.0, norm, out=[], ws=ws)),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_clip_grad_norm(g, 1.0, norm, out=[torch.zeros(7, device="cuda")], ws=ws)),
        (Bd.SV_ERR_INVALID_ARG, lambda: P.sv_clip_grad_norm(g, 1.0, norm, out=[g[0].view(torch.bfloat16)[:8]], ws=ws)),
    ]
    for code, call in cases:
        with pytest.raises(P.SvError) as e:
            call()
        assert e.value.status == code
    with pytest.raises(ValueError):
        P.sv_grad_norm([torch.zeros((4, 4), device="cuda").t()], norm, ws=ws)
    with pytest.raises(ValueError):
        P.sv_grad_norm([torch.zeros(4)], norm, ws=ws)
