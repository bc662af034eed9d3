"""Pins of the sampler's whole-weight oracle: it agrees with the filters in real
numbers, leaves next to nothing open, and turns planted mistakes away. CPU only."""

import numpy as np
import pytest

from oracle import decode_oracle as o


def rows(vocab, seed=1):
    return (np.random.default_rng(seed).standard_normal(vocab) * 2).astype(np.float32)


@pytest.mark.parametrize("vocab", [100, 32000, 128256])
@pytest.mark.parametrize("setting", [(1.0, 0, 0.9, 0.0), (5.0, 0, 0.95, 0.0), (1.4, 6000, 0.97, 0.0), (1.0, 0, 1.0, 0.003), (0.7, 50, 0.8, 0.02)], ids=str)
def test_counts_hold_the_real_ones_and_little_else(vocab, setting):
    l = rows(vocab)
    order, low, high = o.sample_weights(l, setting[0])
    a, b = o.sample_kept(low, high, *setting[1:])
    _, mask, _ = o.sample_filters(l, *setting)
    assert a <= mask.sum() <= b and b - a <= max(1, 0.01 * a)
    assert np.array_equal(np.sort(order[:mask.sum()]), np.flatnonzero(mask))


def test_by_hand():
    l = np.log(np.array([0.1, 0.4, 0.1, 0.25, 0.15]))
    order, low, high = o.sample_weights(l, 1.0)
    assert order.tolist() == [1, 3, 4, 0, 2] and high[0] == 2.0 ** 32 and abs(low[1] - 0.625 * 2.0 ** 32) < 2.0 ** 32 * 2.0 ** -19
    assert o.sample_kept(low, high, 0, 0.6, 0.0) == (2, 2) and o.sample_kept(low, high, 0, 0.66, 0.0) == (3, 3)
    assert o.sample_kept(low, high, 3, 0.6, 0.0) == (2, 2) and o.sample_kept(low, high, 2, 1.0, 0.0) == (2, 2)
    assert o.sample_kept(low, high, 0, 1.0, 0.3) == (3, 3) and o.sample_kept(low, high, 0, -2.0, 0.0) == (1, 1)
    ok = lambda u, t, p, n: o.sample_drawn_ok(order, low, high, 1.0, l, u, t, p, n)  # noqa: E731
    assert ok(0.5, 1, 0.4 / 0.65, 2) and ok(0.7, 3, 0.25 / 0.65, 2) and ok(0.05, 0, 0.1, 5)
    assert not ok(0.7, 1, 0.4 / 0.65, 2) and not ok(0.5, 1, 0.4, 2) and not ok(0.5, 4, 0.15 / 0.65, 2) and not ok(0.7, 3, 0.2500001 / 0.65 * 1.00001, 2)


@pytest.mark.parametrize("vocab", [32000, 128256])
def test_planted_mistakes_are_turned_away(vocab):
    """A cut 1% off, a weight left out of the whole, a draw two places on, a probability of the whole row."""
    l, T, p, u = rows(vocab), 1.0, 0.9, 0.37
    order, low, high = o.sample_weights(l, T)
    a, b = o.sample_kept(low, high, 0, p, 0.0)
    assert not a <= int(1.01 * b) <= b and not a <= int(0.99 * a) <= b
    assert not a <= o.sample_kept(low, high, vocab - vocab // 20, p, 0.0)[0] <= b
    w = np.zeros(vocab)
    w[order[:a]] = (low + high)[:a] / 2
    upto = w.cumsum()
    t = int(np.searchsorted(upto, u * upto[-1], side="right"))
    good = w[t] / upto[-1]
    assert o.sample_drawn_ok(order, low, high, T, l, u, t, good, a)
    kept = np.flatnonzero(w)
    far = int(kept[min(np.searchsorted(kept, t) + max(2, len(kept) // 1000), len(kept) - 1)])
    assert not o.sample_drawn_ok(order, low, high, T, l, u, far, w[far] / upto[-1], a)
    assert not o.sample_drawn_ok(order, low, high, T, l, u, t, good * p, a)
    assert not o.sample_drawn_ok(order, low, high, T, l, u, t, good * (1 + 2.0 ** -14), a)
