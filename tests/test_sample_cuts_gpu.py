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
