"""Pins of the decode operators' oracle: hand-worked values, closed forms and
planted mistakes. CPU only."""

import numpy as np
import pytest

from oracle import decode_oracle as o


def test_kv_quantise_by_hand():
    x = np.zeros((1, 128))
    x[0, 0], x[0, 1], x[0, 2], x[0, 3] = 7.0, -3.5, 2.5, 0.49     # scale 1: ties to even, below half to 0
    x[0, 64], x[0, 65] = -14.0, 3.0                               # scale 2: 1.5 is a tie, to 2
    q, s = o.kv_quantise(x)
    assert s.tolist() == [[1.0, 2.0]]
    assert q[0, :4].tolist() == [7, -4, 2, 0] and q[0, 64:66].tolist() == [-7, 2]
    assert np.array_equal(o.kv_values(q, s)[0, 64:66], [-14.0, 4.0])


def test_kv_quantise_extremes():
    x = np.zeros((4, 64))
    x[1, 5] = np.nan
    x[1, 6] = 7.0
    x[2, 0], x[2, 1] = np.inf, 1.0
    x[3, 0] = 2.0 ** -27                                          # the FP16 scale rounds to 0
    q, s = o.kv_quantise(x)
    assert s[:, 0].tolist() == [0.0, 1.0, 65504.0, 0.0]
    assert not q[0].any() and q[1, 5] == 0 and q[1, 6] == 7 and q[2, 0] == 7 and q[2, 1] == 0 and not q[3].any()


def test_kv_quantise_scale_rounds_before_codes():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((50, 64))
    q, s = o.kv_quantise(x)
    assert np.abs(q).max() == 7
    assert np.all(np.abs(o.kv_values(q, s) - x) <= s.astype(np.float64) * (0.5 + 7 * 2.0 ** -11))


def test_rotate_quarter_turn_and_norm():
    x = np.arange(1.0, 9.0).reshape(1, 1, 8)
    c, s = np.zeros((1, 2)), np.ones((1, 2))                      # 90 degrees, first 4 dimensions: pairs (0, 2), (1, 3)
    assert o.rotate(x, c, s)[0, 0].tolist() == [-3, -4, 1, 2, 5, 6, 7, 8]
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 8))
    a = rng.uniform(0, 6, (3, 4))
    y = o.rotate(x, np.cos(a), np.sin(a), np.float64)
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    assert np.allclose(o.rotate(y, np.cos(a), -np.sin(a), np.float64), x)


def test_attend_closed_forms():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((9, 2, 4)), rng.standard_normal((9, 2, 4))
    out, _, _ = o.attend(np.zeros((3, 4, 4)), k, v, [8, 0, -1], 1.0)
    assert np.allclose(out[0, 0], v[:, 0].mean(0)) and np.allclose(out[0, 3], v[:, 1].mean(0))
    assert np.array_equal(out[1, 1], v[0, 0]) and not out[2].any()
    out, _, _ = o.attend(np.zeros((1, 2, 4)), k, v, [8], 1.0, window=3)
    assert np.allclose(out[0, 1], v[6:9, 1].mean(0))
    out, _, _ = o.attend(np.zeros((1, 2, 4)), k, v, [8], 1.0, window=100)
    assert np.allclose(out[0, 1], v[:, 1].mean(0))
    q = np.zeros((1, 2, 4))
    q[0, 0, 0] = np.log(3.0)                                      # two keys, scores log 3 and 0: weights 3/4, 1/4
    kk = np.zeros((2, 2, 4))
    kk[0, 0, 0] = 1.0
    out, _, _ = o.attend(q, kk, v[:2], [1], 1.0)
    assert np.allclose(out[0, 0], 0.75 * v[0, 0] + 0.25 * v[1, 0])


def test_attend_bound_admits_rounding_and_rejects_a_missing_key():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((1, 2, 64)), rng.standard_normal((40, 1, 64)), rng.standard_normal((40, 1, 64))
    out, spread, reach = o.attend(q, k, v, [39], 0.125)
    ok = lambda g: o.attend_within_bound(g, out, spread, reach, 8 * np.abs(v).max() / 7, 40)  # noqa: E731
    assert ok(out * (1 + 2.0 ** -9)).all()
    for wrong in (o.attend(q, k, v, [38], 0.125)[0], o.attend(q, k, v, [39], 0.126)[0], o.attend(q, k, v, [39], 0.125, 39)[0],
                  -out, np.roll(out, 1, -1)):
        assert not ok(wrong).all()


def test_residual_norm_by_hand():
    out, r = o.residual_norm([[1.0, 5.0]], [[2.0, -1.0]], [1.0, 2.0], 0.0, lambda a: a)
    assert np.allclose(r, [[3.0, 4.0]]) and np.allclose(out, [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]])
    out, _ = o.residual_norm([[0.0, 0.0]], None, [1.0, 1.0], 1e-5, lambda a: a)
    assert not out.any()


def kept(*a):
    return np.flatnonzero(o.sample_filters(*a)[1]).tolist()


def test_sample_filters_by_hand():
    l = np.log([0.1, 0.4, 0.1, 0.25, 0.15])
    assert kept(l, 1.0, 0, 1.0, 0.0) == [0, 1, 2, 3, 4]
    assert kept(l, 1.0, 2, 1.0, 0.0) == [1, 3]
    assert kept([1.0, 2.0, 2.0, 2.0], 1.0, 2, 1.0, 0.0) == [1, 2]          # ties: the lowest indices
    assert kept(l, 1.0, 0, 0.6, 0.0) == [1, 3] and kept(l, 1.0, 0, 0.66, 0.0) == [1, 3, 4]
    assert kept(l, 1.0, 3, 0.6, 0.0) == [1, 3]                              # 0.6 * 0.8 = 0.48 < 0.65
    assert kept(l, 1.0, 3, 0.45, 0.0) == [1]                                # 0.36 < 0.4
    assert kept(l, 1.0, 0, 1.0, 0.3) == [1, 3, 4] and kept(l, 1.0, 0, 0.0, 0.0) == [1]
    assert kept(l, 0.5, 0, 1.0, 0.3) == [1, 3] and kept(l, 0.0, 0, 1.0, 0.0) == [1]
    assert kept([-np.inf, 0.0, np.nan, -np.inf], 1.0, 0, 1.0, 0.0) == [1]
    assert kept([-np.inf, np.inf, 3.0, np.inf], 1.0, 0, 1.0, 0.0) == [1, 2, 3]
    assert kept([-np.inf, np.nan], 1.0, 0, 1.0, 0.0) == []
    e, _, _ = o.sample_filters(l, 2.0, 0, 1.0, 0.0)
    assert np.allclose(e ** 2, np.exp(l) / 0.4)


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9, 0.999])
def test_sample_top_p_is_the_shortest_prefix(p):
    rng = np.random.default_rng(4)
    l = rng.standard_normal(200) * 2
    e, mask, _ = o.sample_filters(l, 1.0, 0, p, 0.0)
    full = np.exp(l - l.max())
    assert full[mask].sum() >= p * full.sum()
    assert full[mask].sum() - full[mask].min() < p * full.sum()
    assert full[mask].min() >= full[~mask].max()
