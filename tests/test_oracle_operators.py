"""Pins of the fp64 definitions of the operators around the decode step: gradients against differences,
identities of the distributions, orders with ties."""
import numpy as np
import pytest

from oracle import operators_oracle as O


def _logits(rng, N, V):
    return (2.0 * rng.standard_normal((N, V))).astype(np.float32)


@pytest.mark.parametrize("T", [1.0, 0.7])
def test_gradient_against_differences(T):
    rng = np.random.default_rng(1)
    N, V = 3, 11
    z = np.round(_logits(rng, N, V) * 1024) / np.float32(1024)      # steps of 2^-7 are exact then
    tok = np.array([4, 0, 10])
    g, h = rng.standard_normal(N), rng.standard_normal(N)

    def value(zz):
        r = O.token_logprobs(zz, tok, T)
        return float((g * r["logprob"] + h * r["entropy"]).sum())

    dz = O.token_logprobs_grad(z, tok, g, h, T)["dz"]
    for r in range(N):
        for v in range(V):
            d = {}
            for s in (2, 1, -1, -2):                        # differences of fourth order
                zz = z.copy()
                zz[r, v] += np.float32(s * 2.0 ** -7)
                d[s] = value(zz)
            est = (8 * (d[1] - d[-1]) - (d[2] - d[-2])) / (12 * 2.0 ** -7)
            assert abs(est - dz[r, v]) < 1e-6, (r, v)


def test_gradients_of_a_row_sum_to_zero():
    rng = np.random.default_rng(2)
    z = _logits(rng, 5, 97)
    out = O.token_logprobs_grad(z, np.array([1, 2, 96, -1, 5]), rng.standard_normal(5), rng.standard_normal(5), 1.3)
    assert np.abs(out["dz"].sum(1)).max() < 1e-12
    assert not out["dz"][3].any()


def test_order_of_equal_logits_is_by_token():
    z = np.array([[1.0, 3.0, 3.0, -np.inf, 1.0, 0.0, -0.0]], np.float32)
    out = O.token_logprobs(z, np.array([4]), n_top=8)
    assert out["top_token"][0].tolist() == [1, 2, 0, 4, 5, 6, -1, -1]
    assert out["rank"][0] == 4
    assert out["top_logprob"][0, 3] == out["logprob"][0]


def test_entropy_and_normaliser_of_known_rows():
    out = O.token_logprobs(np.zeros((1, 8), np.float32), np.array([3]))
    assert np.isclose(out["entropy"][0], np.log(8)) and np.isclose(out["logprob"][0], -np.log(8))
    assert np.isclose(out["lse"][0], np.log(8))
    one = np.full((1, 5), -np.inf, np.float32)
    one[0, 2] = 7.0
    out = O.token_logprobs(one, np.array([2]), n_top=2)
    assert out["logprob"][0] == 0.0 and out["entropy"][0] == 0.0 and out["top_token"][0].tolist() == [2, -1]
    assert O.token_logprobs(one, np.array([1]))["logprob"][0] == -np.inf


@pytest.mark.parametrize("fill", [-np.inf, np.nan, np.inf, -1e30])
def test_bad_rows(fill):
    z = np.full((1, 4), fill, np.float32)
    out = O.token_logprobs(z, np.array([0]), n_top=1)
    assert out["flags"][0] == O.BAD_ROW and np.isnan(out["logprob"][0]) and out["top_token"][0, 0] == -1


def test_embedding_gradient_is_the_transpose_of_the_lookup():
    rng = np.random.default_rng(3)
    V, D, n = 9, 4, 30
    w = rng.standard_normal((V, D)).astype(np.float32)
    ids = rng.integers(-1, V + 1, n)
    g = rng.standard_normal((n, D)).astype(np.float32)
    s, a, c = O.embedding_grad(g, ids, V, 1.5)
    assert np.isclose((O.embedding(w, ids, 1.5) * g).sum(), (s * w).sum())
    assert c.sum() == ((ids >= 0) & (ids < V)).sum() and (a >= np.abs(s) - 1e-12).all()


def test_rounding_and_clipping():
    assert O.to_bf16(np.array([1.0 + 2.0 ** -8, 1.0 + 3 * 2.0 ** -8])).tolist() == [1.0, 1.0 + 2.0 ** -6]
    assert O.grad_norm([np.array([3.0], np.float32), np.array([[4.0]], np.float32)]) == 5.0
    assert O.clip_factor(5.0, 10.0) == 1.0 and O.clip_factor(np.inf, 1.0) == 1.0
    assert np.isclose(O.clip_factor(5.0, 1.0), 0.2)
