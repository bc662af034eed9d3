"""The sampler's cuts and draws: top-p by weight over whole rows, and arguments at
the ends of their ranges."""

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
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
