"""CPU pins of the oracles of the gated projections, the linear cross entropy, the
norms of queries and keys, and dropout: central differences in float64, the
generator's published answers, closed forms."""
import numpy as np
import pytest

from oracle import dropout, gated, linear_ce, logprob, qknorm


def _difference(f, x, d, h=1e-6):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_gradients_by_differences(act):
    rng = np.random.default_rng(0)
    M, N, K = 3, 5, 4
    x, w, b = rng.normal(0, 1, (M, K)), rng.normal(0, 1, (2 * N, K)), rng.normal(0, 1, 2 * N)
    dh = rng.normal(0, 1, (M, N))
    dpre = gated.backward(dh, gated.forward(x, w, b, act)[1], act)
    for arg, grad in (("x", dpre @ w), ("w", dpre.T @ x), ("b", dpre.sum(0))):
        v = {"x": x, "w": w, "b": b}
        d = rng.normal(0, 1, v[arg].shape)
        got = _difference(lambda a: (dh * gated.forward(**{**v, arg: a}, act=act)[0]).sum(), v[arg], d)
        assert abs(got - (grad * d).sum()) <= 1e-7 * (1 + abs(got))


def test_gated_activations():
    x = np.array([-800.0, -3.0, 0.0, 2.0, 50.0])
    a, d = gated.activation("silu", x)
    assert a[0] == 0 and a[2] == 0 and d[2] == 0.5 and a[4] == 50 and d[4] == 1
    assert np.isclose(a[1], -3 / (1 + np.exp(3.0)), rtol=1e-15)
    g, _ = gated.activation("gelu", x)
    assert np.isclose(g[3], 0.5 * 2 * (1 + np.tanh(np.sqrt(2 / np.pi) * (2 + 0.044715 * 8))), rtol=1e-15)


def test_linear_ce_agrees_with_log_probabilities():
    rng = np.random.default_rng(1)
    z, t = rng.normal(0, 3, (6, 11)), np.array([0, 10, -1, 5, 11, 3])
    z[3, 5] = -np.inf
    z[5, :] = -np.inf
    stats, loss = linear_ce.forward(z, t)
    ref, logp, ent, _, _ = logprob.forward(z, t, 0)
    assert np.allclose(stats, ref, rtol=1e-14, atol=1e-14)
    assert np.allclose(loss, -logp, equal_nan=True, rtol=1e-13)
    g = rng.normal(0, 1, 6)
    a = linear_ce.dlogits(z, t, stats, g, 8.0)
    b, _ = logprob.backward(z, t, ref, ent, None, -g, None, None, 8.0)
    assert np.allclose(a, b, equal_nan=True, rtol=1e-12, atol=1e-14)


def test_linear_ce_gradient_by_differences():
    rng = np.random.default_rng(2)
    z, t = rng.normal(0, 2, (4, 7)), np.array([1, -1, 6, 0])
    g = linear_ce.mean_weights(t)
    assert np.allclose(g, 1 / 3)
    f = lambda a: (g * linear_ce.forward(a, t)[1]).sum()
    d = rng.normal(0, 1, z.shape)
    got = _difference(f, z, d)
    assert abs(got - (linear_ce.dlogits(z, t, linear_ce.forward(z, t)[0], g, 1.0) * d).sum()) <= 1e-8


@pytest.mark.parametrize("interleaved", [False, True])
def test_qknorm_gradients_by_differences(interleaved):
    rng = np.random.default_rng(3)
    rows, hq, hk, copy, hd, pairs, base = 3, 2, 1, 1, 10, [2, 2], [100.0, 50.0]
    v = {"x": rng.normal(0, 1, (rows, (hq + hk + copy) * hd)), "wq": rng.normal(1, 0.3, hd),
         "wk": rng.normal(1, 0.3, hd)}
    pos = rng.integers(0, 9, (rows, 2)).astype(float)
    dy = rng.normal(0, 1, v["x"].shape)
    rest = (1e-3, pos, pairs, base, interleaved, hq, hk, hd)
    dx, dwq, dwk, _ = qknorm.backward(v["x"], dy, v["wq"], v["wk"], *rest)
    for arg, grad in (("x", dx), ("wq", dwq), ("wk", dwk)):
        d = rng.normal(0, 1, v[arg].shape)
        got = _difference(lambda a: (dy * qknorm.forward(**{**v, arg: a}, **dict(zip(
            ("eps", "pos", "pairs", "base", "interleaved", "heads_q", "heads_k", "hd"), rest)))[0]).sum(),
            v[arg], d)
        assert abs(got - (grad * d).sum()) <= 1e-7 * (1 + abs(got))


def test_qknorm_has_unit_mean_squares():
    rng = np.random.default_rng(4)
    x = rng.normal(0, 7, (5, 3 * 8))
    y, n = qknorm.forward(x, None, None, 0.0, np.zeros((5, 1)), [3], [10.0], False, 2, 0, 8)
    assert np.allclose((n.reshape(5, 3, 8)[:, :2] ** 2).mean(-1), 1.0)
    assert np.array_equal(y[:, 16:], x[:, 16:]) and np.array_equal(y, n)   # position 0


@pytest.mark.parametrize("counter, key, answer", [
    ([0] * 4, [0] * 2, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
     "d16cfe09 94fdcceb 5001e420 24126ea1")])
def test_philox_published_answers(counter, key, answer):
    """The known answers that the generator's authors publish with it."""
    got = dropout.philox([np.array([c]) for c in counter], key)
    assert " ".join("%08x" % int(v[0]) for v in got) == answer


def test_dropout_keeps_the_right_share():
    n = 1 << 18
    for p in (0.0, 0.1, 0.5, 0.9):
        k, scale = dropout.kept(n, p, 12345678901234567, 3, 2)
        q = np.rint(p * 65536) / 65536
        assert abs((~k).mean() - q) <= 5 * np.sqrt(q * (1 - q) / n) and np.isclose(scale, 1 / (1 - q))
    a, b = (dropout.kept(n, 0.5, 1, s, 2)[0] for s in (0, 1))
    assert abs((a == b).mean() - 0.5) <= 5 * 0.5 / np.sqrt(n)
    assert np.array_equal(dropout.kept(100, 0.5, 9, 9, 9, first=64)[0], dropout.kept(164, 0.5, 9, 9, 9)[0][64:])
