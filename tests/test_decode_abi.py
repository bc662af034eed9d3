"""Refusals of the decode operators: bad arguments are answered on the host,
before anything is enqueued, by the C ABI and by the binding. CPU only."""

import ctypes

import pytest
import torch

import paper_2607_02893_gb300 as vbq
from paper_2607_02893_gb300.decode import _CacheStruct


@pytest.fixture(scope="module")
def lib():
    from paper_2607_02893_gb300 import build
    build.build()
    return vbq.load()


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(4096)
    p.keep = buf
    return (ctypes.addressof(buf) + 15) // 16 * 16


def cache(p, n=4, heads=2, d=64):
    c = _CacheStruct(p, n, heads, d)
    return ctypes.byref(c)


def test_page_bytes(lib):
    assert vbq.vbq_kv_page_bytes(1, 64) == 64 * (2 * 32 + 4)
    assert vbq.vbq_kv_page_bytes(8, 128) == 8 * 64 * (2 * 64 + 8)
    out = ctypes.c_size_t()
    for h, d in ((0, 64), (1025, 64), (1, 96), (1, 512), (1, 0)):
        assert lib.vbq_kv_page_bytes(h, d, ctypes.byref(out)) == -2
    assert lib.vbq_kv_page_bytes(1, 64, None) == -1


def append(lib, p, c=None, table=0, ts=4, tp=4, pos=0, b=1, r=1, q=None, qs=0, h=0, k=0, ks=128, v=0, vs=128, ty=1, cos=None, sin=None,
           rot=0, rr=0, qo=None):
    at = lambda x: p if x == 0 else x  # noqa: E731
    return lib.vbq_kv_append(cache(p) if c is None else c, at(table), ts, tp, at(pos), b, r, q, qs, h, at(k), ks, at(v), vs, ty, cos, sin,
                             rot, rr, qo, None)


def test_append_refusals(lib, p):
    assert lib.vbq_kv_append(None, p, 4, 4, p, 1, 1, None, 0, 0, p, 128, p, 128, 1, None, None, 0, 0, None, None) == -1
    for c, want in ((cache(None), -1), (cache(p, n=0), -1), (cache(p, n=1 << 31), -1), (cache(p, heads=0), -2), (cache(p, d=80), -2),
                    (cache(p + 8), -5)):
        assert append(lib, p, c=c) == want
    assert append(lib, p, table=None) == -1 and append(lib, p, pos=None) == -1
    assert append(lib, p, k=None) == -1 and append(lib, p, v=None) == -1
    assert append(lib, p, b=-1) == -1 and append(lib, p, r=-1) == -1 and append(lib, p, tp=0) == -1 and append(lib, p, ts=-1) == -1
    assert append(lib, p, b=1 << 16, r=1 << 15) == -7
    assert append(lib, p, ty=2) == -1
    assert append(lib, p, q=p, qs=128, h=2) == -1 and append(lib, p, qo=p) == -1
    assert append(lib, p, q=p, qs=128, h=0, qo=p) == -2
    assert append(lib, p, cos=p, rot=32, rr=9) == -1
    for rot in (0, 8, 24, 80):
        assert append(lib, p, cos=p, sin=p, rot=rot, rr=9) == -2
    assert append(lib, p, cos=p, sin=p, rot=32, rr=0) == -1
    assert append(lib, p, r=2, ks=127) == -1 and append(lib, p, r=2, vs=64) == -1
    assert append(lib, p, r=2, ks=130) == -5 and append(lib, p, r=2, ty=0, vs=132) == -5
    assert append(lib, p, k=p + 4) == -5 and append(lib, p, table=p + 2) == -5 and append(lib, p, cos=p + 4, sin=p, rot=32, rr=9) == -5
    assert append(lib, p, b=0) == 0 and append(lib, p, r=0) == 0      # nothing to do


def test_read_and_attend_refusals(lib, p):
    assert lib.vbq_kv_read(None, p, 4, 4, p, 1, 1, p, p, None) == -1
    assert lib.vbq_kv_read(cache(p), None, 4, 4, p, 1, 1, p, p, None) == -1
    assert lib.vbq_kv_read(cache(p), p, 4, 4, p, 1, 1, p + 4, p, None) == -5
    assert lib.vbq_kv_read(cache(p), p, 4, 4, p, 0, 1, p, p, None) == 0 and lib.vbq_kv_read(cache(p), p, 4, 4, p, 1, 1, None, None, None) == 0
    out = ctypes.c_size_t()
    size = lambda c, b, r, h: lib.vbq_kv_workspace_bytes(c, b, r, h, ctypes.byref(out))  # noqa: E731
    assert size(None, 1, 1, 2) == -1 and size(cache(p), -1, 1, 2) == -1 and size(cache(p), 1, 1, 3) == -2 and size(cache(p), 1, 1, 0) == -2
    assert size(cache(p), 1, 17, 2) == -7 and size(cache(p), 1, 0, 2) == -7 and size(cache(p), 1025, 1, 2) == -7 and size(cache(p), 1, 1, 130) == -7
    assert lib.vbq_kv_workspace_bytes(cache(p), 1, 1, 2, None) == -1

    def attend(c=None, b=1, r=1, h=2, scale=1.0, window=0, q=p, o=p, w=p, tp=4):
        return lib.vbq_kv_attend(cache(p) if c is None else c, p, 4, tp, p, b, r, q, h, scale, window, o, w, 1 << 30, None)

    assert attend(c=cache(None)) == -1 and attend(q=None) == -1 and attend(o=None) == -1 and attend(w=None) == -1
    assert attend(h=3) == -2 and attend(r=17) == -7 and attend(b=1025) == -7 and attend(h=130) == -7
    for scale in (float("nan"), float("inf"), -float("inf")):
        assert attend(scale=scale) == -1
    assert attend(window=-1) == -1 and attend(tp=0) == -1
    assert attend(q=p + 2) == -5 and attend(o=p + 8) == -5 and attend(w=p + 8) == -5
    assert attend(b=0) == 0


def test_norm_refusals(lib, p):
    def norm(x=p, xt=1, r=p, rt=1, w=p, eps=1e-5, rows=1, width=64, o=p, ro=p):
        return lib.vbq_residual_norm(x, xt, r, rt, w, eps, rows, width, o, ro, None)

    assert norm(x=None) == -1 and norm(w=None) == -1 and norm(o=None) == -1 and norm(r=None) == -1 and norm(ro=None) == -1
    assert norm(xt=2) == -1 and norm(rt=-1) == -1
    for eps in (-1e-9, float("inf"), float("nan")):
        assert norm(eps=eps) == -1
    assert norm(rows=-1) == -2 and norm(width=0) == -2 and norm(width=(1 << 20) + 1) == -7 and norm(rows=1 << 40, width=2) == -7
    assert norm(x=p + 4) == -5 and norm(w=p + 8) == -5
    assert norm(rows=0) == 0


def test_sample_refusals(lib, p):
    def sample(l=p, stride=100, ty=1, b=2, vocab=100, t=p, k=p, tp=p, mp=p, u=p, o=p, pr=None, ke=None):
        return lib.vbq_sample(l, stride, ty, b, vocab, t, k, tp, mp, u, o, pr, ke, None)

    for name in ("l", "t", "k", "tp", "mp", "u", "o"):
        assert sample(**{name: None}) == -1
    assert sample(ty=3) == -1 and sample(b=-1) == -1 and sample(b=65536) == -7 and sample(vocab=0) == -2
    assert sample(vocab=(1 << 18) + 1, stride=1 << 20) == -7 and sample(stride=99) == -1
    assert sample(l=p + 2) == -5 and sample(l=p + 1, ty=0) == -5 and sample(u=p + 2) == -5 and sample(ke=p + 1) == -5
    assert sample(b=0) == 0


def test_binding_refuses_what_the_library_cannot_see(lib):
    f = torch.zeros
    c = vbq.KvCache(2, 1, 64, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        vbq.vbq_kv_append(c, f(1, 1, dtype=torch.int32), f(1, 1, dtype=torch.int32), f(1, 1, 1, 64), f(1, 1, 1, 64))
    with pytest.raises(ValueError, match="table"):
        vbq.vbq_kv_append(c, f(1, 1), f(1, 1, dtype=torch.int32), f(1, 1, 1, 64), f(1, 1, 1, 64))
    with pytest.raises(ValueError, match="pos"):
        vbq.vbq_kv_read(c, f(1, 1, dtype=torch.int32), f(2, 1, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        vbq.vbq_residual_norm(f(2, 8), None, f(8), 1e-5)
    with pytest.raises(ValueError, match="GPU"):
        vbq.vbq_sample(f(1, 8), f(1), f(1, dtype=torch.int32), f(1), f(1), f(1))
    with pytest.raises(ValueError):
        vbq.KvCache(2, 1, 64, pages=f(100, dtype=torch.uint8))
    with pytest.raises(vbq.VbqError):
        vbq.KvCache(2, 1, 65, device="cpu")
