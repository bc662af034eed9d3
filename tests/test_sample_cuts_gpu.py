"""The sampler's cuts and draws: top-p by weight over whole rows, and arguments at
the ends of their ranges."""

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import decode_oracle as o
from test_norm_sample_gpu import _draw

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 1000, 20000, 128256])
def test_top_p_below_zero_keeps_one_token(vocab):
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy(rng.standard_normal((6, vocab)).astype(np.float32))
    x[5] = 0.25                                                   # all alike: the first
    for top_p in (0.0, -0.25, -2.0, -1e6, float("-inf"), float("nan")):
        for top_k in (0, 3):
            tok, prob, kept, _ = _draw(x, top_p=top_p, top_k=top_k, u=0.99)
            assert kept.tolist() == [1] * 6 and prob.tolist() == [1.0] * 6, (top_p, top_k)
            assert np.array_equal(tok, x.numpy().argmax(1)), (top_p, top_k)


@pytest.mark.parametrize("temperature", [1e-30, 1.0, 1e30, 3e36, 1e38, 3e38, float("inf")])
def test_infinite_logits_share_the_draw_at_any_temperature(temperature):
    """exp((l - inf) / T) is 0 for a finite l however large T is."""
    inf = float("inf")
    x = torch.tensor([[0.0, inf, 3e38, inf, -inf], [5.0, -3e38, 1.0, inf, inf]])
    for u, want in ((0.0, [1, 3]), (0.49, [1, 3]), (0.51, [3, 4]), (0.999, [3, 4])):
        for over in ({}, {"top_p": 0.9}, {"top_k": 3}, {"min_p": 0.01}):
            tok, prob, _, _ = _draw(x, temperature=temperature, u=u, **over)
            assert tok.tolist() == want and prob.tolist() == [0.5, 0.5], (u, over)
    many = torch.full((1, 20000), 7.0)
    many[0, 15001::2] = inf                                       # 2500 of them
    tok, prob, kept, _ = _draw(many, temperature=temperature, u=0.5, top_p=0.5)
    assert kept[0] == 1250 and tok[0] == 15001 + 2 * 625 and abs(prob[0] * 1250 - 1) < 1e-6


def _check(logits, sharp=0.01, **over):
    """Every row against the whole-weight oracle; nothing is skipped. The oracle's own width, how far it leaves the count
    open, may be one token or `sharp` of them. Returns the counts."""
    tok, prob, kept, p = _draw(logits, **over)
    rows = logits.float().numpy()
    for b in range(rows.shape[0]):
        T, k, top_p, mp, u = (p[n][b] for n in ("temperature", "top_k", "top_p", "min_p", "u"))
        order, low, high = o.sample_weights(rows[b], T)
        least, most = o.sample_kept(low, high, int(k), float(top_p), float(mp))
        assert most - least <= max(1, sharp * least), f"row {b}: the oracle leaves {least}..{most}"
        assert least <= kept[b] <= most, f"row {b}: {kept[b]} kept, not {least}..{most}"
        assert o.sample_drawn_ok(order, low, high, T, rows[b], float(u), int(tok[b]), float(prob[b]), int(kept[b])), f"row {b}"
    return kept


SETTINGS = {
    "top_p": {"top_p": 0.9}, "top_p_each": {"top_p": [0.05, 0.5, 0.99, 0.9999]}, "hot": {"top_p": 0.95, "temperature": 5.0},
    "cold": {"top_p": 0.9, "temperature": 0.5}, "top_k_wide": {"top_k": 6000, "top_p": 0.97}, "top_k": {"top_k": 300, "top_p": 0.8},
    "min_p": {"min_p": 0.003}, "all_three": {"top_k": 20000, "top_p": 0.98, "min_p": 0.0005, "temperature": 1.4}, "none": {},
    "top_k_alone": {"top_k": [1, 255, 5000, 30000]},
}


@pytest.mark.parametrize("vocab", [3000, 4097, 16384, 32000, 50257, 128256, 151937, 1 << 18])
@pytest.mark.parametrize("setting", sorted(SETTINGS))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_every_row_of_a_wide_nucleus(vocab, setting, dtype):
    """A head's logits: a wide bulk and some tokens above it; BF16 has equal ones by the thousand."""
    rng = np.random.default_rng(vocab + 7 * sorted(SETTINGS).index(setting))
    x = rng.standard_normal((4, vocab)).astype(np.float32) * 2
    x[:, rng.integers(0, vocab, 40)] += rng.uniform(2, 6, 40).astype(np.float32)
    kept = _check(torch.from_numpy(x).to(dtype), u=torch.from_numpy(rng.random(4).astype(np.float32)), **SETTINGS[setting])
    if setting == "top_p":
        assert kept.min() > 256                                   # the path that cuts a row too long for one block's list


@pytest.mark.parametrize("batch", [9, 16, 24, 25])
def test_every_row_of_a_batch(batch):
    """Batches that take clusters of 6 and of 8."""
    rng = np.random.default_rng(batch)
    x = torch.from_numpy(rng.standard_normal((batch, 128256)).astype(np.float32) * 2)
    _check(x, u=torch.from_numpy(rng.random(batch).astype(np.float32)), top_p=0.9)


@pytest.mark.parametrize("vocab", [20000, 128256])
@pytest.mark.parametrize("spread", [0.0, 1e-7, 1e-3, 0.02])
@pytest.mark.parametrize("base", [0.0, 7.0])
def test_cuts_by_weight_among_near_equal_logits(vocab, spread, base):
    """Thousands of logits in one bin of the histogram: the cut is found inside it."""
    rng = np.random.default_rng(vocab + int(base))
    x = (rng.integers(-300, 300, (5, vocab)) * spread / 300).astype(np.float32) + np.float32(base)
    _check(torch.from_numpy(x), u=torch.from_numpy(rng.random(5).astype(np.float32)), top_p=[0.1, 0.3, 0.5, 0.7, 0.9])
    _check(torch.from_numpy(x), u=torch.from_numpy(rng.random(5).astype(np.float32)), top_k=vocab // 3, top_p=0.5, min_p=0.5)


@pytest.mark.parametrize("u", [0.0, 2.0 ** -30, 0.25, 0.5, 1 - 2.0 ** -24])
def test_draws_at_the_ends(u):
    rng = np.random.default_rng(3)
    _check(torch.from_numpy(rng.standard_normal((4, 32000)).astype(np.float32)), u=u, top_p=[0.3, 0.9, 0.999, 1.0])


@pytest.mark.parametrize("vocab", [20000, 32000, 151937])
@pytest.mark.parametrize("batch", [8, 14, 15, 16, 17, 22, 23, 24, 28, 40])
def test_batches_about_the_changes_of_cluster_size(vocab, batch):
    rng = np.random.default_rng([vocab, batch])
    x = torch.from_numpy(rng.standard_normal((batch, vocab)).astype(np.float32) * 2)
    u = torch.from_numpy(rng.random(batch).astype(np.float32))
    _check(x, u=u, top_p=0.9)
    _check(x, u=u, top_k=40, top_p=0.95, temperature=0.8)
