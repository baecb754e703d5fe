"""The example that serves and fits: its gradients against torch's own in float64, and that the companion
gets closer to the target."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("entropy_weight", [0.0, 0.3])
def test_gradients(entropy_weight):
    """A float32 chain of products over D = 32 and V = 500 terms of either sign: 1e-5 of a gradient's norm is some
    twenty times the rounding of its sums."""
    from paper_2509_24328_amd import companion_fit as C
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    V, D, N = 500, 32, 70
    m = C.Model(V, D, gen)
    contexts = torch.randint(0, V, (N,), generator=gen, device="cuda", dtype=torch.int32)
    contexts[:20] = contexts[0]
    tokens = torch.randint(0, V, (N,), generator=gen, device="cuda", dtype=torch.int32)
    tokens[5:9] = -1
    fit = C.Fit(m, N, entropy_weight=entropy_weight)
    fit.gradients(contexts, tokens)
    table, layer = (p.double().cpu().requires_grad_() for p in fit.params)
    c, t = contexts.long().cpu(), tokens.long().cpu()
    z = m.gain * (torch.tanh(table[c] * m.scale @ layer) @ table.t())
    lp = torch.log_softmax(z, -1)
    on = t >= 0
    loss = -lp[on, t[on]].mean() - entropy_weight * -(lp.exp() * lp).sum(-1)[on].mean()
    loss.backward()
    for g, p in zip(fit.grads, (table, layer)):
        assert (g.double().cpu() - p.grad).norm() <= 1e-5 * p.grad.norm()


def test_the_companion_gets_closer():
    from paper_2509_24328_amd import companion_fit as C
    log = C.run(V=512, D=32, B=64, k=4, steps=80, seed=1)
    first, last = log[0], log[-1]
    assert all(abs(v) < 1e6 for r in log for v in r.values())
    assert last["companion"] > first["companion"] + 0.1
    assert last["similarity"] > first["similarity"]
