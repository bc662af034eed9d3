"""Append and read, bit by bit against the oracle, from seeds that are the same in
every process."""

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import decode_oracle as o
from test_kv_gpu import _held, _table

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("rot", [0, 16, 64])
def test_append_from_fixed_seeds(seed, d, bf16, rot):
    rng = np.random.default_rng([seed, d, bf16, rot])
    heads, hk = [(4, 4), (6, 3), (8, 1), (5, 5)][seed]
    lens = [int(n) for n in rng.integers(1, 300, 1 + seed)]
    rows = min(1 + 5 * seed, min(lens))
    table, pages = _table(lens, rng)
    cache = vbq.KvCache(pages, hk, d)
    cache.pages.fill_(0xff)
    dtype = [torch.float32, torch.bfloat16][bf16]
    fused = torch.from_numpy((rng.standard_normal((len(lens), rows, heads + 2 * hk, d)) * 10.0 ** rng.uniform(-4, 4)).astype(np.float32)).to(DEV).to(dtype)
    pos = np.stack([rng.permutation(n)[:rows] for n in lens]).astype(np.int32)
    pos[rng.random(pos.shape) < 0.2] = -1
    cos = sin = None
    if rot:
        angle = rng.uniform(-9, 9, (300, rot // 2))
        cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    ct, st = (None if a is None else torch.from_numpy(a).to(DEV) for a in (cos, sin))
    pt = torch.from_numpy(pos).to(DEV)
    q_out = vbq.vbq_kv_append(cache, table, pt, fused[:, :, heads:heads + hk], fused[:, :, heads + hk:], q=fused[:, :, :heads], cos=ct, sin=st)
    kr, vr = vbq.vbq_kv_read(cache, table, pt)
    x = fused.float().cpu().numpy().reshape(-1, heads + 2 * hk, d)
    flat = pos.reshape(-1)
    if rot:
        at = np.maximum(flat, 0)
        x[:, :heads + hk] = o.rotate(x[:, :heads + hk], cos[at], sin[at])
    live = (flat >= 0)[:, None, None]
    for got, part in ((kr, x[:, heads:heads + hk]), (vr, x[:, heads + hk:])):
        want = np.where(live, _held(part)[0], 0.0).astype(np.float32)
        assert np.array_equal(got.cpu().numpy().reshape(want.shape), want)
    want = torch.from_numpy(np.where(live, x[:, :heads], 0.0).astype(np.float32)).to(torch.bfloat16)
    assert torch.equal(q_out.cpu().reshape(want.shape), want)
    assert vbq.vbq_device_status() is None
