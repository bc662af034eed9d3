"""Refusals and marshalling of the linear-attention operators: bad arguments are
answered on the host, before anything is enqueued, by the C ABI and by the
binding. CPU only."""

import contextlib
import ctypes
from types import SimpleNamespace

import pytest
import torch

import paper_2607_02893_gb300 as vbq
from paper_2607_02893_gb300 import decode, delta
from paper_2607_02893_gb300.delta import _SequencesStruct

F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


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


def seq(starts=None, slots=None, fresh=None, batch=2, rows=3, tokens=6):
    return ctypes.byref(_SequencesStruct(starts, slots, fresh, batch, rows, tokens))


def refused_sequences(call, p):
    assert call(None) == -1
    for s, want in ((seq(batch=-1), -1), (seq(rows=-1), -1), (seq(tokens=-1), -1), (seq(tokens=5), -1), (seq(batch=65536, rows=0, tokens=0), -7),
                    (seq(starts=p, tokens=1 << 31), -7), (seq(starts=p + 2), -5), (seq(slots=p + 1), -5), (seq(fresh=p + 2), -5)):
        assert call(s) == want
    for s in (seq(batch=0, tokens=0), seq(rows=0, tokens=0), seq(starts=p, tokens=0)):
        assert call(s) == 0                                       # nothing to do


def test_conv_refusals(lib, p):
    def conv(s=None, x=p, xs=64, ty=1, w=p, b=None, taps=4, c=64, st=p, n=2, silu=1, o=p):
        return lib.vbq_causal_conv(s, x, xs, ty, w, b, taps, c, st, n, silu, o, None)

    refused_sequences(conv, p)
    ok = seq()
    for taps in (0, 1, 5):
        assert conv(ok, taps=taps) == -7
    for c in (0, 4, 60, (1 << 20) + 8):
        assert conv(ok, c=c) == -2
    for name in ("x", "w", "st", "o"):
        assert conv(ok, **{name: None}) == -1
        assert conv(ok, **{name: p + 8}) == -5
    assert conv(ok, b=p + 4) == -5 and conv(ok, ty=2) == -1 and conv(ok, n=0) == -1 and conv(ok, n=1 << 31) == -1 and conv(ok, silu=2) == -1
    assert conv(ok, xs=63) == -1 and conv(ok, xs=66) == -5 and conv(ok, xs=68, ty=0) == -5


def test_delta_refusals(lib, p):
    def rule(s=None, st=p, n=2, q=p, qs=128, k=p, ks=128, v=p, vs=256, ty=0, hk=2, dk=64, h=4, dv=64, d=p, ds=4, b=p, bs=4, gt=1, a=None, dt=None,
             scale=1.0, norm=1, o=p):
        return lib.vbq_delta_rule(s, st, n, q, qs, k, ks, v, vs, ty, hk, dk, h, dv, d, ds, b, bs, gt, a, dt, scale, norm, o, None)

    refused_sequences(rule, p)
    ok = seq()
    for change in (dict(dk=32), dict(dk=256), dict(dv=32), dict(dv=96), dict(h=3), dict(h=0), dict(hk=0), dict(h=2048)):
        assert rule(ok, **change) == -2
    for name in ("st", "q", "k", "v", "d", "b", "o"):
        assert rule(ok, **{name: None}) == -1
    for name in ("st", "q", "k", "v", "o"):
        assert rule(ok, **{name: p + 8}) == -5
    for change in (dict(ty=2), dict(gt=-1), dict(n=0), dict(a=p), dict(dt=p), dict(norm=2), dict(scale=float("nan")), dict(scale=float("inf")),
                   dict(qs=127), dict(ks=64), dict(vs=255), dict(ds=3), dict(bs=0)):
        assert rule(ok, **change) == -1
    for change in (dict(qs=132), dict(vs=260), dict(d=p + 2), dict(b=p + 1), dict(d=p + 1, gt=0), dict(a=p + 2, dt=p)):
        assert rule(ok, **change) == -5


def test_gated_norm_refusals(lib, p):
    def norm(x=p, xs=128, xt=0, z=p, zs=128, zt=1, w=p, eps=1e-6, rows=2, h=2, width=64, o=p):
        return lib.vbq_gated_norm(x, xs, xt, z, zs, zt, w, eps, rows, h, width, o, None)

    for eps in (-1e-9, float("inf"), float("nan")):
        assert norm(eps=eps) == -1
    for change in (dict(width=0), dict(width=60), dict(width=264), dict(h=0), dict(h=1025), dict(rows=-1)):
        assert norm(**change) == -2
    for name in ("x", "w", "o"):
        assert norm(**{name: None}) == -1
    assert norm(xt=2) == -1 and norm(zt=2) == -1 and norm(xs=127) == -1 and norm(zs=64) == -1 and norm(rows=1 << 31) == -7
    assert norm(x=p + 8) == -5 and norm(z=p + 8) == -5 and norm(w=p + 4) == -5 and norm(xs=132) == -5 and norm(zs=130) == -5
    assert norm(rows=0) == 0 and norm(rows=0, z=None, zt=9) == 0


class Fake:
    """A tensor of `shape` at a made-up address on a GPU, dense but for the elements between its rows."""
    made = 0

    def __init__(self, *shape, dtype=F32, device=0, row=None):
        Fake.made += 1
        self.shape, self.dtype, self.at, self.index, self.row = shape, dtype, Fake.made << 24, device, row
        self.device = SimpleNamespace(type="cuda", index=device)

    def stride(self):
        out, n = [], 1
        for s in reversed(self.shape):
            out.insert(0, n)
            n *= s
        if self.row:
            out[0] = self.row
        return tuple(out)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def is_contiguous(self): return self.row is None              # noqa: E704
    def get_device(self): return self.index                       # noqa: E704
    def data_ptr(self): return self.at                            # noqa: E704


STREAM = 64


@pytest.fixture
def calls(monkeypatch):
    """The calls that reached the library: (name, arguments)."""
    from paper_2607_02893_gb300 import build
    build.build()
    log, keep = [], {}
    names = ("vbq_causal_conv", "vbq_delta_rule", "vbq_gated_norm")
    for name in ("vbq_kv_append", "vbq_kv_read", "vbq_kv_attend", "vbq_residual_norm", "vbq_sample") + names:
        kind = ctypes.CFUNCTYPE(*vbq.SIGNATURES[name][:1], *vbq.SIGNATURES[name][1])
        keep[name] = kind(lambda *a, name=name: log.append((name, a)) or 0)
    monkeypatch.setattr(decode._b, "load", lambda: SimpleNamespace(**keep))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    decode._load()
    delta._load()
    yield log
    monkeypatch.undo()
    decode._load()                                                # the real entry points again
    delta._load()


def sequences(device=0, tokens=6):
    return vbq.Sequences(2, 3, starts=Fake(3, dtype=I32, device=device), tokens=tokens, slots=Fake(2, dtype=I32, device=device))


def conv(s=None, **change):
    a = dict(x=Fake(6, 64, row=100), weight=Fake(64, 4), state=Fake(5, 3, 64), bias=Fake(64), out=Fake(6, 64, dtype=BF16)) | change
    return vbq.vbq_causal_conv(s or sequences(), a["x"], a["weight"], a["state"], bias=a["bias"], out=a["out"], stream=STREAM)


def rule(s=None, **change):
    b = lambda *shape, **k: Fake(*shape, dtype=BF16, **k)  # noqa: E731
    a = dict(state=Fake(5, 4, 64, 128), q=b(6, 2, 64, row=1000), k=b(6, 2, 64, row=1008), v=b(6, 4, 128, row=1016), decay=Fake(6, 4, row=9),
             beta=Fake(6, 4, row=11), a_log=Fake(4), dt_bias=Fake(4), scale=None, out=b(6, 4, 128)) | change
    return vbq.vbq_delta_rule(s or sequences(), a["state"], a["q"], a["k"], a["v"], a["decay"], a["beta"], a_log=a["a_log"], dt_bias=a["dt_bias"],
                              scale=a["scale"], out=a["out"], stream=STREAM)


def gated(**change):
    a = dict(x=Fake(6, 4, 64, dtype=BF16), gate=Fake(6, 4, 64, row=600), weight=Fake(64), out=Fake(6, 4, 64, dtype=BF16)) | change
    return vbq.vbq_gated_norm(a["x"], a["gate"], a["weight"], 1e-6, out=a["out"], stream=STREAM)


def test_arguments_arrive(calls):
    s = sequences()
    x, w, st, bias, out = Fake(6, 64, row=100), Fake(64, 4), Fake(5, 3, 64), Fake(64), Fake(6, 64, dtype=BF16)
    conv(s, x=x, weight=w, state=st, bias=bias, out=out)
    assert calls[0][1] == (s._address, x.at, 100, 1, w.at, bias.at, 4, 64, st.at, 5, 1, out.at, STREAM)
    assert (s._struct.starts, s._struct.slots, s._struct.fresh) == (s.starts.at, s.slots.at, None)
    assert (s._struct.batch, s._struct.rows, s._struct.tokens) == (2, 3, 6)
    rule(s)
    a = calls[1][1]
    assert a[0] == s._address and a[2] == 5 and (a[4], a[6], a[8]) == (1000, 1008, 1016) and a[9:14] == (0, 2, 64, 4, 128)
    assert (a[15], a[17], a[18]) == (9, 11, 1) and a[19] and a[20] and a[21:23] == (0.125, 1) and a[24] == STREAM
    rule(a_log=None, dt_bias=None, scale=0.5)
    a = calls[2][1]
    assert a[19:22] == (None, None, 0.5)
    gated()
    a = calls[3][1]
    assert (a[1], a[2], a[4], a[5]) == (256, 0, 600, 1) and a[8:11] == (6, 4, 64)
    gated(gate=None)
    assert calls[4][1][3] is None


def test_shapes_types_and_devices_are_refused(calls):
    b = lambda *shape, **k: Fake(*shape, dtype=BF16, **k)  # noqa: E731
    for change in (dict(x=Fake(5, 64)), dict(x=Fake(6, 64, dtype=I32)), dict(x=Fake(6, 64, 1)), dict(weight=Fake(63, 4)), dict(weight=b(64, 4)),
                   dict(state=Fake(5, 4, 64)), dict(state=Fake(5, 3, 64, row=999)), dict(state=Fake(3, 64)), dict(bias=Fake(63)), dict(out=Fake(6, 64)),
                   dict(out=b(5, 64)), dict(state=Fake(5, 3, 64, device=1))):
        with pytest.raises(ValueError):
            conv(**change)
    for change in (dict(state=Fake(5, 4, 128, 64)), dict(state=b(5, 4, 64, 128)), dict(q=b(6, 2, 128)), dict(k=b(6, 1, 64)), dict(q=Fake(6, 2, 64)),
                   dict(v=b(5, 4, 128)), dict(decay=Fake(6, 2)), dict(beta=b(6, 4)), dict(a_log=None), dict(dt_bias=None), dict(a_log=Fake(3)),
                   dict(out=b(6, 4, 64)), dict(out=Fake(6, 4, 128)), dict(k=b(6, 2, 64, device=1))):
        with pytest.raises(ValueError):
            rule(**change)
    for change in (dict(x=b(6, 64)), dict(gate=Fake(5, 4, 64)), dict(gate=Fake(6, 4, 32)), dict(weight=Fake(32)), dict(out=Fake(6, 4, 64)), dict(weight=b(64))):
        with pytest.raises(ValueError):
            gated(**change)
    there = sequences(device=1)
    for call in (lambda: conv(there), lambda: rule(there), lambda: conv(x=Fake(6, 64, device=1)), lambda: gated(x=b(6, 4, 64, device=1))):
        with pytest.raises(ValueError):
            call()
    assert calls == []


def test_sequences_are_refused(lib):
    i = lambda n: Fake(n, dtype=I32)  # noqa: E731
    for call in (lambda: vbq.Sequences(-1, 2), lambda: vbq.Sequences(2, 1 << 31), lambda: vbq.Sequences(2, 3, tokens=5), lambda: vbq.Sequences(2, 3, starts=i(3)),
                 lambda: vbq.Sequences(2, 3, starts=i(2), tokens=6), lambda: vbq.Sequences(2, 3, slots=i(3)), lambda: vbq.Sequences(2, 3, slots=Fake(2)),
                 lambda: vbq.Sequences(2, 3, fresh=torch.zeros(2, dtype=I32)), lambda: vbq.Sequences(2, 3, slots=i(2), fresh=Fake(2, dtype=I32, device=1)),
                 lambda: vbq.Sequences(2, 3, slots=Fake(2, dtype=I32, row=2))):
        with pytest.raises(ValueError):
            call()
    assert vbq.Sequences(2, 3, tokens=6).tokens == 6 and vbq.Sequences(2, 3).device == -1
    f = torch.zeros
    with pytest.raises(ValueError, match="GPU"):
        vbq.vbq_causal_conv(vbq.Sequences(1, 2), f(2, 8), f(8, 4), f(1, 3, 8))
    with pytest.raises(ValueError, match="GPU"):
        vbq.vbq_delta_rule(vbq.Sequences(1, 2), f(1, 1, 64, 64), f(2, 1, 64), f(2, 1, 64), f(2, 1, 64), f(2, 1), f(2, 1))
    with pytest.raises(ValueError, match="GPU"):
        vbq.vbq_gated_norm(f(2, 1, 64), None, f(64), 1e-6)


@pytest.mark.parametrize("stream", [4096, SimpleNamespace(cuda_stream=8192), None], ids=["handle", "object", "current"])
def test_outputs_are_made_on_the_call_s_stream(monkeypatch, stream):
    on, current, streams = [], [None], []

    @contextlib.contextmanager
    def under(s):
        before, current[0] = current[0], s
        yield
        current[0] = before

    monkeypatch.setattr(torch, "empty", lambda shape, **k: on.append(current[0]) or Fake(*shape, dtype=BF16))
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
    call = lambda *a: streams.append(a[-1]) or 0  # noqa: E731
    monkeypatch.setattr(delta, "_native", SimpleNamespace(conv=call, delta=call, gated=call))
    s = sequences()
    vbq.vbq_causal_conv(s, Fake(6, 64), Fake(64, 4), Fake(5, 3, 64), stream=stream)
    vbq.vbq_delta_rule(s, Fake(5, 4, 64, 64), Fake(6, 2, 64), Fake(6, 2, 64), Fake(6, 4, 64), Fake(6, 4), Fake(6, 4), stream=stream)
    vbq.vbq_gated_norm(Fake(6, 4, 64), None, Fake(64), 1e-6, stream=stream)
    handle = stream if stream is None or isinstance(stream, int) else stream.cuda_stream
    assert on == [handle] * 3 and streams == [stream] * 3
