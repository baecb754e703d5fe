"""sv_sample's nucleus over rows that rise with the token, as long as a call takes them.

Every vector of such a row raises the largest entry that a lane has seen.  With u = 0 the token is the first one that is kept: of a row
that rises, the one at which the nucleus ends.  top_p lies 4e-6 to 4e-5 of the mass beside that of the entries above some value,
where a mass that is not as exact as it claims ends the nucleus at another token."""
import numpy as np
import pytest
import torch

import paper_2509_24328_amd as P
import test_gpu_sample as S

pytestmark = pytest.mark.gpu


def kept_from(z, top_p):
    """First token kept of a rising row of different values (fp64), and how near the decision was, relative to the mass."""
    w = np.exp(z - z.max())
    above = w[::-1].cumsum()[::-1]                       # mass from a token on
    target = float(np.float32(top_p)) * above[0]
    first = int(np.flatnonzero(above >= target)[-1])
    near = min(above[first] - target, target - (above[first + 1] if first + 1 < len(z) else 0.0))
    # (equal values are kept together)
    return int(np.searchsorted(z, z[first])), near / above[0]


@pytest.mark.parametrize("V", [1 << 20, 1 << 22, (1 << 24) - 5])
@pytest.mark.parametrize("top", [0.02, 0.4])
def test_where_the_nucleus_of_a_rising_row_ends(V, top):
    z = torch.linspace(0.0, top, V, dtype=torch.float64).float()
    zd = z.double().numpy()
    w = np.exp(zd - zd.max())
    total, zg = w.sum(), z.cuda()[None]
    u = torch.zeros(1, dtype=torch.float64, device="cuda")
    token = torch.zeros(1, dtype=torch.int32, device="cuda")
    decided = 0
    for part in (0.25, 0.5, 0.75):
        beside = w[zd >= np.float32(part) * np.float32(zd.max())].sum() / total
        for off in (-4e-5, -2.4e-5, -1.2e-5, -6e-6, 6e-6, 1.2e-5, 2.4e-5, 4e-5):
            top_p = float(np.float32(beside + off))
            want, near = kept_from(zd, top_p)
            if near < V * 2.0 ** -53:                     # (a sum's rounding here)
                continue
            decided += 1
            P.sv_sample(zg, u, token, top_p=top_p)
            assert token.item() == want, (part, off, token.item(), want, near)
    assert decided >= 20


@pytest.mark.parametrize("V", [1 << 20, 1 << 22, (1 << 24) - 5])
@pytest.mark.parametrize("spikes", [3, 300])
def test_a_few_large_entries_over_a_rising_row(V, spikes):
    """The nucleus ends among entries that weigh half the row."""
    z = torch.linspace(0.0, 0.05, V, dtype=torch.float64)
    each = np.log(z.exp().sum().item() / spikes)         # (together as much as the rest)
    at = torch.arange(spikes) * (V // spikes // 2) + 100
    z[at] = each + 1e-3 * torch.arange(spikes, dtype=torch.float64)
    z = z.float()
    zd = z.double().numpy()
    w = np.exp(zd - zd.max())
    total, zg = w.sum(), z.cuda()[None]
    u = torch.zeros(1, dtype=torch.float64, device="cuda")
    token = torch.zeros(1, dtype=torch.int32, device="cuda")
    order = at.numpy()[::-1]                              # by falling value
    for n in {1, 2, spikes // 2, spikes - 1}:
        for off in (-2e-5, -1e-5, -6e-6, 6e-6, 1e-5, 2e-5):
            top_p = float(np.float32(w[order[:n]].sum() / total + off))
            target = top_p * total
            run = w[order].cumsum()
            many = int((run < target).sum()) + 1          # entries kept: until their mass reaches the target
            assert many <= spikes and np.abs(run - target).min() > 1e-9 * total
            P.sv_sample(zg, u, token, top_p=top_p)
            assert token.item() == order[:many].min(), (n, off, token.item(), order[:many].min())


@pytest.mark.parametrize("base", [2.0 ** 21, 2.0 ** 23, -2.0 ** 23, 2.0 ** 29, -2.0 ** 29])
@pytest.mark.parametrize("temperature", [1.0, 0.7, 30.0])
def test_logits_far_from_zero(base, temperature):
    """Logits of up to 2^29, several of their steps apart, of rising, falling and mixed rows."""
    V, step = 20000, max(abs(base) * 2.0 ** -23, 2.0 ** -6)
    g = torch.Generator().manual_seed(3)
    z = base + step * torch.randint(0, 40, (6, V), generator=g).double()
    z[1], z[2] = z[1].sort().values, z[2].sort(descending=True).values
    z[3:, torch.randint(0, V, (30,), generator=g)] += 60 * step
    u = torch.rand(6, generator=g, dtype=torch.float64).cuda()
    for warp in (dict(top_p=0.9), dict(top_p=0.5, min_p=0.01), dict(top_k=50, top_p=0.9), dict()):
        S.check(z.float().cuda(), u, near=1, temperature=temperature, **warp)
