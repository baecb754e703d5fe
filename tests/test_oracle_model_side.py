"""Pins of the oracle of the model side of a step: worked numbers and identities."""
import numpy as np

from oracle import model_side_oracle as O


def test_rotation_by_hand():
    f = np.array([np.pi / 2, 0.0])
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    assert np.allclose(O.turned(x, [1], f), [[[-3.0, 2.0, 1.0, 4.0, 5.0]]])
    assert np.allclose(O.turned(x, [1], f, pairs=True), [[[-2.0, 1.0, 3.0, 4.0, 5.0]]])
    y = np.random.default_rng(0).standard_normal((3, 2, 10))
    g = O.frequencies(6)
    assert np.allclose(O.turned(O.turned(y, [3, 0, 9], g), [3, 0, 9], g, inverse=True), y)
    # scores depend on distances alone
    q, k = y[:1, :1], y[1:2, :1]
    s = [float((O.turned(q, [p + 5], g) * O.turned(k, [p], g)).sum()) for p in (0, 7, 100)]
    assert np.allclose(s, s[0])


def test_frequencies():
    assert np.allclose(O.frequencies(4, 100.0), [1.0, 0.1])
    assert np.allclose(O.frequencies(4, 100.0, 1, 2.0), [0.5, 0.05])
    assert np.allclose(O.frequencies(4, 100.0, 2, 3.0), [1.0, 1.0 / 30.0])      # the slowest pair: divided by the factor
    f = O.frequencies(4, 1e4, 3, 4.0, 1.0, 4.0, 200)                            # 31.8 turns: stays; 0.318: divided
    assert np.allclose(f, [1.0, 0.01 / 4.0])


def test_e4m3():
    v = O.e4m3(np.arange(128, dtype=np.uint8))
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1.0 and v[0x7E] == 448.0 and np.isnan(v[0x7F])
    assert (np.diff(v[:127]) > 0).all()


def test_attention_by_hand():
    k = np.zeros((2, 1, 2, 8))
    v = np.arange(32, dtype=float).reshape(2, 1, 2, 8)
    q = np.ones((2, 1, 8))
    out, lse, flags, _, _ = O.attention(q, k, v, [1], np.array([[1, 0]]), None, 2, 1.0)
    assert np.allclose(out[0, 0], (v[1, 0, 0] + v[1, 0, 1]) / 2) and np.allclose(lse[:, 0], np.log([2.0, 3.0]))
    assert np.allclose(out[1, 0], (v[1, 0, 0] + v[1, 0, 1] + v[0, 0, 0]) / 3) and not flags.any()
    out, lse, flags, _, _ = O.attention(q, k, v, [1], np.array([[1, 7]]), None, 2, 1.0, window=1, first=[2])
    assert (out[0] == 0).all() and lse[0, 0] == -np.inf and flags.tolist() == [0, 256]


def test_draw_by_hand():
    z = np.log(np.array([1.0, 2.0, 4.0, 2.0, 1.0]))
    assert [O.draw(z, u)[0] for u in (0.0, 0.05, 0.15, 0.5, 0.75, 0.95)] == [0, 0, 1, 2, 3, 4]
    assert [O.draw(z, u, top_k=2)[0] for u in (0.0, 0.3, 0.8)] == [1, 2, 3]      # two values tie for the second place
    assert [O.draw(z, u, top_p=0.375)[0] for u in (0.0, 0.99)] == [2, 2]
    assert [O.draw(z, u, top_p=0.5)[0] for u in (0.0, 0.99)] == [1, 3]
    assert [O.draw(z, u, min_p=0.3)[0] for u in (0.0, 0.99)] == [1, 3]
    assert np.isclose(O.draw(z, 0.0, top_k=1)[1], 0.0) and O.draw(np.array([np.nan]), 0.0)[0] == -1
