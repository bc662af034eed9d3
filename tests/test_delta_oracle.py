"""Pins of the linear-attention oracle: cases whose answers are known without it."""

import numpy as np
import pytest

from oracle import delta_oracle as o


def test_one_token_from_nothing():
    """S = 0: u = beta v, S = beta k v^T, o = scale (q.k) beta v."""
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((1, 2, 8)), rng.standard_normal((1, 2, 8)), rng.standard_normal((1, 4, 6))
    g, beta = -rng.random((1, 4)), rng.random((1, 4))
    out, s, _, _ = o.delta_rule(q, k, v, g, beta, np.zeros((4, 8, 6)), 0.5, normalize=False)
    for h in range(4):
        qq, kk = q[0, h // 2], k[0, h // 2]
        assert np.allclose(s[h], beta[0, h] * np.outer(kk, v[0, h]), rtol=1e-14)
        assert np.allclose(out[0, h], 0.5 * beta[0, h] * (qq @ kk) * v[0, h], rtol=1e-13)


def test_overwrites_a_key():
    """beta 1, unit key, no decay: what the state holds for the key becomes v, what it holds for keys across it stays."""
    rng = np.random.default_rng(1)
    e = np.eye(8)
    s0 = rng.standard_normal((1, 8, 5))
    v = rng.standard_normal((1, 1, 5))
    _, s, _, _ = o.delta_rule(e[2][None, None], e[2][None, None], v, np.zeros((1, 1)), np.ones((1, 1)), s0, 1.0, normalize=False)
    assert np.allclose(s[0, 2], v[0, 0])
    assert np.array_equal(np.delete(s[0], 2, 0), np.delete(s0[0], 2, 0))


def test_linear_map_form():
    """S_t = e^g (1 - beta k k^T) S_{t-1} + beta k v^T, as matrices."""
    rng = np.random.default_rng(2)
    n, d, dv = 150, 8, 4
    q, k, v = rng.standard_normal((n, 1, d)), rng.standard_normal((n, 1, d)), rng.standard_normal((n, 1, dv))
    g, beta = -0.1 * rng.random((n, 1)), rng.random((n, 1))
    s0 = rng.standard_normal((1, d, dv))
    out, s, _, _ = o.delta_rule(q, k, v, g, beta, s0, 0.3)
    m = s0[0].copy()
    for t in range(n):
        u = k[t, 0] / np.sqrt(k[t, 0] @ k[t, 0] + 1e-6)
        m = np.exp(g[t, 0]) * (np.eye(d) - beta[t, 0] * np.outer(u, u)) @ m + beta[t, 0] * np.outer(u, v[t, 0])
        w = q[t, 0] / np.sqrt(q[t, 0] @ q[t, 0] + 1e-6) * 0.3
        assert np.allclose(out[t, 0], w @ m, rtol=1e-9, atol=1e-12)
    assert np.allclose(s[0], m, rtol=1e-9, atol=1e-12)


def test_a_planted_mistake_is_outside_the_bound():
    """A decay applied after the update instead of before it, and a key head off by one."""
    rng = np.random.default_rng(3)
    n, d = 70, 64
    q, k, v = rng.standard_normal((n, 2, d)), rng.standard_normal((n, 2, d)), rng.standard_normal((n, 4, d))
    g, beta = -0.05 * rng.random((n, 4)), rng.random((n, 4))
    s0 = rng.standard_normal((4, d, d))
    out, s, ob, sb = o.delta_rule(q, k, v, g, beta, s0, d ** -0.5)
    for wrong in (o.delta_rule(q, k[:, ::-1], v, g, beta, s0, d ** -0.5), o.delta_rule(q, k, v, np.roll(g, 1, 0), beta, s0, d ** -0.5)):
        assert (np.abs(wrong[0] - out) > ob + 2.0 ** -8 * np.abs(out)).mean() > 0.3
        assert (np.abs(wrong[1] - s) > sb).mean() > 0.3


@pytest.mark.parametrize("rows", [1, 2, 3, 9])
def test_conv_carries_its_inputs(rows):
    """Cut anywhere, a sequence gives the same; against a direct sum."""
    rng = np.random.default_rng(rows)
    x, w, past, bias = rng.standard_normal((rows + 5, 8)), rng.standard_normal((8, 4)), rng.standard_normal((3, 8)), rng.standard_normal(8)
    y, last, _ = o.causal_conv(x, w, past, bias, False)
    a, mid, _ = o.causal_conv(x[:rows], w, past, bias, False)
    b, end, _ = o.causal_conv(x[rows:], w, mid, bias, False)
    assert np.allclose(np.concatenate((a, b)), y) and np.array_equal(end, last)
    line = np.concatenate((past, x))
    assert np.allclose(y[2, 5], sum(w[5, j] * line[2 + j, 5] for j in range(4)) + bias[5])


def test_gates_and_norm():
    g, b = o.gates(np.array([[0.0, 5.0, -500.0]]), np.array([[0.0, 1.0, -1.0]]), np.log(np.array([2.0, 1.0, 1.0])), np.zeros(3))
    assert np.allclose(g, [[-2 * np.log(2), -np.log1p(np.exp(5)), 0.0]]) and np.allclose(b[0, 0], 0.5)
    g, b = o.gates(np.array([[3.0, -200.0]]), np.array([[1.5, 0.0]]))
    assert g.tolist() == [[0.0, -100.0]] and b.tolist() == [[1.5, 0.0]]
    y = o.gated_norm(np.full((1, 4), 3.0), np.zeros((1, 4)), np.ones(4), 0.0)
    assert not y.any()
    assert np.allclose(o.gated_norm(np.full((1, 4), -3.0), None, np.arange(4.0), 0.0), -np.arange(4.0))
