"""The decode binding's own refusals: tensors whose type, size, strides or device
the C ABI cannot see are turned away before a call is made, and refused calls
leave their outputs alone. Accepted: BF16 bit patterns, streams by object or handle."""

import gc

import pytest
import torch

import paper_2607_02893_gb300 as vbq

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


def _cache():
    cache = vbq.KvCache(3, 2, 64)
    cache.pages.zero_()
    return cache, torch.tensor([[0, 1, 2]], dtype=I32, device=DEV), torch.tensor([[5, 6]], dtype=I32, device=DEV)


def test_cache_calls_refuse_wrong_tensors():
    cache, table, pos = _cache()
    k = torch.randn(1, 2, 2, 64, device=DEV)
    q = torch.randn(1, 2, 4, 64, device=DEV)
    cos = torch.ones(64, 16, device=DEV)
    out = torch.full((1, 2, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    before = cache.pages.clone()
    bad = [
        dict(table=table.long()), dict(table=table[0]), dict(table=table.cpu()), dict(table=torch.zeros(1, 6, dtype=I32, device=DEV)[:, ::2]),
        dict(pos=pos.long()), dict(pos=pos[0]), dict(pos=pos.cpu()), dict(pos=torch.zeros(2, 2, dtype=I32, device=DEV)),
        dict(pos=torch.zeros(1, 4, dtype=I32, device=DEV)[:, ::2]),
        dict(k=k.double()), dict(k=k.half()), dict(k=k.to(torch.bfloat16)), dict(k=k[:, :1]), dict(k=k[:, :, :1]), dict(k=k.cpu()), dict(k=k[0]),
        dict(k=k.transpose(2, 3).contiguous().transpose(2, 3)), dict(k=torch.randn(1, 2, 2, 128, device=DEV)[..., ::2]),
        dict(q=q[..., :32]), dict(q=q.to(torch.bfloat16)), dict(q_out=out[:, :1]), dict(q_out=out.float()), dict(q_out=out.cpu()),
        dict(cos=cos.double()), dict(cos=cos[:, ::2]), dict(sin=cos[:32]), dict(cos=cos.cpu()), dict(cos=cos[0]),
    ]
    for change in bad:
        args = dict(table=table, pos=pos, k=k, v=k, q=q, cos=cos, sin=cos, q_out=out) | change
        with pytest.raises(ValueError):
            vbq.vbq_kv_append(cache, args["table"], args["pos"], args["k"], args["v"], q=args["q"], cos=args["cos"], sin=args["sin"],
                              q_out=args["q_out"])
    torch.cuda.synchronize()
    assert torch.equal(cache.pages, before) and bool((out == 7).all())
    qb = q.to(torch.bfloat16)
    ws = vbq.vbq_kv_workspace(cache, 1, 2, 4)
    for args in ((q, out, ws), (qb[:, :1], out, ws), (qb[0], out, ws), (qb.cpu(), out, ws), (qb, out[:, :1], ws), (qb, out.float(), ws),
                 (qb, out, ws.cpu()), (qb, out, ws[::2])):
        with pytest.raises(ValueError):
            vbq.vbq_kv_attend(cache, table, pos, args[0], out=args[1], workspace=args[2])
    with pytest.raises(vbq.VbqError):
        vbq.vbq_kv_attend(cache, table, pos, qb, out=out, workspace=ws[:16])
    with pytest.raises(vbq.VbqError):
        vbq.vbq_kv_attend(cache, table, pos, torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16, device=DEV), workspace=ws)
    with pytest.raises((ValueError, OverflowError)):
        vbq.vbq_kv_attend(cache, table, pos, qb, out=out, workspace=ws, window=1 << 40)
    for o in (out, torch.empty(1, 2, 2, 32, device=DEV), torch.empty(1, 2, 2, 64)):
        with pytest.raises(ValueError):
            vbq.vbq_kv_read(cache, table, pos, k_out=o)
    torch.cuda.synchronize()
    assert bool((out == 7).all())


def test_norm_and_sample_refuse_wrong_tensors():
    x, w = torch.randn(4, 64, device=DEV), torch.ones(64, device=DEV)
    o = torch.empty(4, 64, dtype=torch.bfloat16, device=DEV)
    for args in ((x.half(), None, w, o), (x.cpu(), None, w, o), (x.t(), None, w, o), (x, x.cpu(), w, o), (x, x[:2], w, o), (x, x.half(), w, o),
                 (x, None, w[:32], o), (x, None, w.to(torch.bfloat16), o), (x, None, w, x), (x, None, w, o[:2])):
        with pytest.raises(ValueError):
            vbq.vbq_residual_norm(args[0], args[1], args[2], 1e-5, out=args[3])
    with pytest.raises(ValueError):
        vbq.vbq_residual_norm(x, x, w, 1e-5, residual_out=x.to(torch.bfloat16))
    with pytest.raises(TypeError):
        vbq.vbq_residual_norm(x, None, w, "eps")
    l, f, i = torch.randn(2, 100, device=DEV), torch.ones(2, device=DEV), torch.ones(2, dtype=I32, device=DEV)
    good = [l, f, i, f, f, f * 0.5]
    for at, t in ((0, l.half()), (0, l.cpu()), (0, l.t()), (0, l[0]), (1, f[:1]), (1, f.double()), (2, f), (2, i.long()), (3, i), (5, f.cpu())):
        args = list(good)
        args[at] = t
        with pytest.raises(ValueError):
            vbq.vbq_sample(*args)
    for name, t in (("tokens", f), ("probs", i), ("kept", i.long()), ("tokens", i[:1])):
        with pytest.raises(ValueError):
            vbq.vbq_sample(*good, **{name: t})


def test_bit_patterns_streams_and_references():
    x, w = torch.randn(3, 128, device=DEV), torch.rand(128, device=DEV)
    want, _ = vbq.vbq_residual_norm(x, None, w, 1e-5)
    bits = torch.empty(3, 128, dtype=torch.int16, device=DEV)
    vbq.vbq_residual_norm(x, None, w, 1e-5, out=bits)
    assert torch.equal(bits, want.view(torch.int16))
    a, _ = vbq.vbq_residual_norm(want.view(torch.int16), None, w, 1e-5)
    assert torch.equal(a, vbq.vbq_residual_norm(want, None, w, 1e-5)[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for s in (side, side.cuda_stream):
        out = torch.zeros_like(want)
        side.wait_stream(torch.cuda.current_stream())
        vbq.vbq_residual_norm(x, None, w, 1e-5, out=out, stream=s)
        side.synchronize()
        assert torch.equal(out, want)
    deep, _ = vbq.vbq_residual_norm(x.reshape(1, 1, 3, 1, 128), None, w, 1e-5)
    assert deep.shape == (1, 1, 3, 1, 128) and torch.equal(deep.reshape(3, 128), want)
    import sys
    gc.collect()
    before = [sys.getrefcount(t) for t in (x, w, want, torch.float32, torch.bfloat16)]
    for _ in range(200):
        vbq.vbq_residual_norm(x, None, w, 1e-5, out=want)
        with pytest.raises(ValueError):
            vbq.vbq_residual_norm(x, None, w[:5], 1e-5, out=want)
    after = [sys.getrefcount(t) for t in (x, w, want, torch.float32, torch.bfloat16)]
    assert all(abs(i - j) < 20 for i, j in zip(before, after))
