"""The decoding example: its steps against the same computation in fp64, graph
replays against eager steps, and the command itself."""

import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import decode_oracle as o

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


def _weights(layout, spec):
    w = torch.empty(spec.n, spec.k, device="cuda")
    vbq.vbq_dequant(layout, w_out=w)
    return w.double().cpu().numpy()


def _bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("batch", [1, 3])
def test_steps_match_fp64(batch):
    """Three steps of two layers of the 131M-class stack. The reference rounds to BF16 where the step does and holds
    keys and values in 4 bits; its inputs to each rounding differ by earlier roundings (2^-9 at some ten places, and
    now and then a key or value a 4-bit step away), so logits agree to a few percent of their norm: 5% is allowed."""
    from decode import Decoder
    dec = Decoder("stack131m", batch, max_tokens=64, layers=2)
    ws = [_weights(lay, s) for lay, s in zip(dec.layouts, dec.specs)]
    norms = [w.double().cpu().numpy() for w in dec.weights]
    emb = dec.embedding.double().cpu().numpy()
    cos, sin = dec.cos.cpu().numpy(), dec.sin.cpu().numpy()
    h, hk, d = dec.heads, dec.kv_heads, dec.head_dim
    keys = [[[] for _ in range(batch)] for _ in range(2)]
    vals = [[[] for _ in range(batch)] for _ in range(2)]
    dec.reset(torch.arange(5, 5 + batch, dtype=torch.int32, device="cuda"))
    for step in range(3):
        dec.u.fill_(0.3 + 0.2 * step)
        first = dec.tokens.cpu().numpy()
        dec.step()
        r = emb[first]
        x = _bf16(o.residual_norm(r, None, norms[0], 1e-5, None)[0])
        for layer in range(2):
            qkv = (x @ ws[4 * layer].T).reshape(batch, h + 2 * hk, d)
            c, s = np.repeat(cos[step:step + 1], batch, 0), np.repeat(sin[step:step + 1], batch, 0)
            turned = o.rotate(qkv[:, :h + hk], c, s, np.float64)
            q = _bf16(turned[:, :h])
            att = np.zeros((batch, h, d))
            for b in range(batch):
                keys[layer][b].append(o.kv_values(*o.kv_quantise(turned[b, h:])))
                vals[layer][b].append(o.kv_values(*o.kv_quantise(qkv[b, h + hk:])))
                att[b] = o.attend(q[b][None], np.stack(keys[layer][b]), np.stack(vals[layer][b]), [step], d ** -0.5)[0][0]
            y = _bf16(att).reshape(batch, -1) @ ws[4 * layer + 1].T
            out, r = o.residual_norm(y, r, norms[2 * layer + 1], 1e-5, lambda a: a)
            gu = _bf16(out) @ ws[4 * layer + 2].T
            hid = gu[:, 0::2] / (1 + np.exp(-gu[:, 0::2])) * gu[:, 1::2]
            out, r = o.residual_norm((hid if batch == 1 else _bf16(hid)) @ ws[4 * layer + 3].T, r, norms[2 * layer + 2], 1e-5,
                                     lambda a: a)
            x = _bf16(out)
        ref = x @ ws[-1].T
        got = dec.logits.double().cpu().numpy()
        assert np.linalg.norm(got - ref) <= 0.05 * np.linalg.norm(ref), f"step {step}"
        tok = dec.tokens.cpu().numpy()
        for b in range(batch):                                    # the draw, from the step's own logits
            e, mask, _ = o.sample_filters(got[b], 0.8, 50, float(np.float32(0.95)), 0.0)
            assert mask[tok[b]]
    assert dec.pos.flatten().tolist() == [3] * batch
    vbq.vbq_device_status()


def test_graph_replays_match_eager_steps():
    """The split-K products add in a varying order, so a step's logits vary in their last bits; the tokens drawn with the same
    random numbers agree until such a bit decides one."""
    from decode import Decoder
    dec = Decoder("stack131m", 1, max_tokens=128, layers=3)
    u = torch.rand(40, 1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    first = torch.tensor([11], dtype=torch.int32, device="cuda")
    graph = dec.capture()
    a, b = dec.generate(first, u, graph), dec.generate(first, u)
    assert torch.equal(a[:4], b[:4])
    assert int((a >= 0).all()) and int((a < dec.vocab).all())


def test_command_runs():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "decode.py"), "--layers", "2", "--tokens", "8", "--batch", "2"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert "tokens/s" in r.stdout
