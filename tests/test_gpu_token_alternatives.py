"""Alternatives where they lie together: in few lanes of a workgroup (entries whose vectors are a workgroup's
lanes apart), at the start or end of a row, in ascending or descending order, and where almost nothing has mass."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P

pytestmark = pytest.mark.gpu


def check(z, n_top):
    N, V = z.shape
    top = torch.full((N, n_top), -777, dtype=torch.int32, device="cuda")
    val = torch.full((N, n_top), 5.0, device="cuda")
    lse = torch.empty(N, device="cuda")
    P.sv_token_logprobs(z.cuda(), None, None, lse, None, None, top, val)
    z64 = z.double()
    order = z64.sort(dim=-1, descending=True, stable=True).indices[:, :n_top]
    lp = (z64 - z64.logsumexp(-1, keepdim=True)).gather(1, order)
    want = torch.full((N, n_top), -1, dtype=torch.int32)
    want[:, :order.shape[1]] = order.int().masked_fill(lp == -float("inf"), -1)
    assert np.array_equal(top.cpu().numpy(), want.numpy())
    got = val.cpu().double()[:, :order.shape[1]]
    fin = torch.isfinite(lp)
    assert torch.equal(got[~fin], lp[~fin])
    assert ((got - lp)[fin].abs() <= 2e-6 + 1.3e-7 * lp[fin].abs()).all()
    assert (val.cpu()[:, order.shape[1]:] == -float("inf")).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lanes", [256, 512, 1024])
@pytest.mark.parametrize("wide", [1, 7, 40])
def test_large_entries_in_few_lanes(dtype, lanes, wide):
    """wide lanes hold all large entries: thousands of them in the widest case."""
    V = 400003
    per_vec = 4 if dtype == torch.float32 else 8
    g = torch.Generator().manual_seed(lanes + wide)
    z = torch.randn((2, V), generator=g)
    vec = torch.arange(V) // per_vec
    z[:, vec % lanes < wide] += 20.0
    for n_top in (1, 20, 32):
        check(z.to(dtype), n_top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [5, 31, 32, 33, 255, 2049, 16384, 100001])
def test_orders(dtype, V):
    g = torch.Generator().manual_seed(V)
    up = torch.arange(V).float() * (12.0 / V)
    few = torch.full((V,), -float("inf"))
    few[torch.randperm(V, generator=g)[:4]] = torch.randn(4, generator=g)
    two = torch.where(torch.rand(V, generator=g) < 0.5, 1.0, 2.0)
    first = torch.zeros(V)
    first[:3] = 9.0
    last = torch.zeros(V)
    last[-3:] = 9.0
    z = torch.stack([up, up.flip(0), few, two, first, last, torch.zeros(V)]).to(dtype)
    for n_top in (1, 2, 17, 32):
        check(z, n_top)
