"""Layouts of logits that the scoring calls take: positions picked out of a tensor, dimensions of one, wider rows, and packed
logits without a row."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
from oracle import operators_oracle as O
from test_gpu_token_logprobs import bits, check_grad, logits, same, score

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("at", [slice(0, 1), slice(-1, None), slice(1, 2), -1, slice(0, 4), slice(0, 4, 2)])
@pytest.mark.parametrize("pad", [0, 3])
def test_positions_of_a_batch(dtype, at, pad):
    """One position of each sequence, with and without its dimension, every other one, and all."""
    B, Pn, V = 3, 4, 203
    wide = logits(B * Pn, V + pad, dtype, 9).view(B, Pn, V + pad)
    z = wide.cuda()[:, at, :V]
    want = wide[:, at, :V].reshape(-1, V)
    tok = torch.randint(0, V, z.shape[:-1], generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    same(score(z, tok.cuda(), 3), O.token_logprobs(bits(want), tok.numpy().ravel(), 1.0, 3), 3)
    g = torch.ones(tok.numel())
    dz = torch.full((B, Pn, V + 2), 9.0, dtype=dtype, device="cuda")
    out = dict(logprob=torch.empty(len(g), device="cuda"), entropy=torch.empty(len(g), device="cuda"),
               flags=torch.empty(len(g), dtype=torch.int32, device="cuda"), dz=dz[:, at, :V])
    P.sv_token_logprobs_grad(z, tok.cuda(), g.cuda(), out["dz"], None, out["logprob"], out["entropy"], out["flags"])
    out["dz"] = out["dz"].reshape(-1, V)
    check_grad(want, tok.ravel(), g, None, 1.0, out)
    assert (dz[..., V:] == 9.0).all() and int((dz == 9.0).sum()) >= dz.numel() - len(g) * V


def test_dimensions_of_one():
    V = 64
    z = logits(6, V + 1, F32, 4)
    dev = z.cuda()[:, :V]
    tok = torch.arange(6, dtype=torch.int32)
    ref = O.token_logprobs(bits(z[:, :V]), tok.numpy(), 1.0, 2)
    for view in (dev.unsqueeze(1), dev.unsqueeze(0), dev.unsqueeze(0).unsqueeze(2), dev.unsqueeze(1).unsqueeze(1)):
        same(score(view, tok.view(view.shape[:-1]).cuda(), 2), ref, 2)


def test_layouts_refused():
    z = torch.zeros((4, 6, 8), device="cuda")
    f, tok = torch.zeros(12, device="cuda"), torch.zeros(12, dtype=torch.int32, device="cuda")
    for bad in (z[:, :3], z[:, 0:1, :6].expand(4, 3, 6), z.transpose(0, 1)[:3], z[:2, :, ::2], z.transpose(1, 2)[:, :3]):
        with pytest.raises(ValueError):
            n = bad.numel() // bad.shape[-1]
            P.sv_token_logprobs(bad, tok.new_zeros(n), f.new_zeros(n))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_packed_logits_without_a_row(dtype):
    """No position is there (a step in which every sequence has ended); offsets that say otherwise point at bad rows."""
    B, Pn, V = 3, 2, 50
    z = torch.empty((0, V), dtype=dtype, device="cuda")
    tok = torch.ones((B, Pn), dtype=torch.int32, device="cuda")
    got = score(z, tok, 2, offsets=torch.zeros(B + 1, dtype=torch.int32, device="cuda"))
    for k in ("logprob", "lse", "entropy", "rank", "flags"):
        assert not got[k].any(), k
    assert (got["top_token"] == -1).all() and (got["top_logprob"] == -np.inf).all()
    got = score(z, tok, 2, offsets=torch.tensor([0, 1, 1, 1], dtype=torch.int32, device="cuda"))
    assert got["flags"].tolist() == [[1, 0], [0, 0], [0, 0]] and np.isnan(got["logprob"][0, 0])
