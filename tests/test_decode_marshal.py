"""What the binding's marshalling passes on and what it refuses. CPU only:
tensors that only say where they are, and entry points that only write down
their arguments."""

import ctypes
from types import SimpleNamespace

import pytest
import torch

import paper_2607_02893_gb300 as vbq
from paper_2607_02893_gb300 import decode

F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32
STREAM = 64


class Fake:
    """A dense tensor of `shape` at a made-up address on a GPU."""
    made = 0

    def __init__(self, *shape, dtype=F32, device=0):
        Fake.made += 1
        self.shape, self.dtype, self.at, self.index = shape, dtype, Fake.made << 20, device
        self.device = SimpleNamespace(type="cuda", index=device)
        n = 1
        for s in shape:
            n *= s
        self.count, self.nbytes = n, 4 * n

    def stride(self):
        out, n = [], 1
        for s in reversed(self.shape):
            out.insert(0, n)
            n *= s
        return tuple(out)

    def numel(self): return self.count                            # noqa: E704
    def is_contiguous(self): return True                          # noqa: E704
    def get_device(self): return self.index                       # noqa: E704
    def data_ptr(self): return self.at                            # noqa: E704


@pytest.fixture
def calls(monkeypatch):
    """The calls that reached the library: (name, arguments)."""
    from paper_2607_02893_gb300 import build
    build.build()
    lib, log, keep = vbq.load(), [], {}
    for name in ("vbq_kv_append", "vbq_kv_read", "vbq_kv_attend", "vbq_residual_norm", "vbq_sample"):
        kind = ctypes.CFUNCTYPE(*vbq.SIGNATURES[name][:1], *vbq.SIGNATURES[name][1])
        keep[name] = kind(lambda *a, name=name: log.append((name, a)) or 0)
    monkeypatch.setattr(decode._b, "load", lambda: SimpleNamespace(**keep))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    decode._load()
    yield log
    monkeypatch.undo()
    assert decode._b.load() is lib
    decode._load()                                                # the real entry points again


def cache(device=0):
    c = vbq.KvCache.__new__(vbq.KvCache)
    c._struct = decode._CacheStruct(1 << 40, 4, 2, 64)
    c._address, c.device, c.kv_heads, c.head_dim = ctypes.addressof(c._struct), device, 2, 64
    return c


def append(**change):
    a = dict(table=Fake(1, 4, dtype=I32), pos=Fake(1, 2, dtype=I32), k=Fake(1, 2, 2, 64), v=Fake(1, 2, 2, 64), q=Fake(1, 2, 4, 64),
             cos=Fake(100, 32), sin=Fake(100, 32), q_out=Fake(1, 2, 4, 64, dtype=BF16), stream=STREAM) | change
    return vbq.vbq_kv_append(cache(), a["table"], a["pos"], a["k"], a["v"], q=a["q"], cos=a["cos"], sin=a["sin"], q_out=a["q_out"],
                             stream=a["stream"])


def norm(**change):
    a = dict(x=Fake(3, 64), residual=Fake(3, 64, dtype=BF16), weight=Fake(64), out=Fake(3, 64, dtype=BF16),
             residual_out=Fake(3, 64, dtype=BF16)) | change
    return vbq.vbq_residual_norm(a["x"], a["residual"], a["weight"], 1e-5, out=a["out"], residual_out=a["residual_out"], stream=STREAM)


def test_arguments_that_go_together(calls):
    """One without the other is what the C call refuses; the binding must not drop it and go on."""
    for change in (dict(cos=None), dict(sin=None)):
        with pytest.raises(ValueError, match="cos and sin"):
            append(**change)
    with pytest.raises(ValueError, match="q and q_out"):
        append(q=None)
    with pytest.raises(ValueError, match="residual and residual_out"):
        norm(residual=None)
    assert calls == []
    append()
    append(cos=None, sin=None)
    append(q=None, q_out=None)
    norm()
    norm(residual=None, residual_out=None)
    assert [c[0] for c in calls] == ["vbq_kv_append"] * 3 + ["vbq_residual_norm"] * 2


def test_arguments_arrive(calls):
    q, k, cos, sin, q_out = Fake(1, 2, 4, 64), Fake(1, 2, 2, 64), Fake(100, 16), Fake(100, 16), Fake(1, 2, 4, 64, dtype=BF16)
    append(q=q, k=k, cos=cos, sin=sin, q_out=q_out)
    a = calls[0][1]
    assert (a[2], a[3], a[5], a[6]) == (4, 4, 1, 2)               # table stride, its pages, batch, rows
    assert (a[7], a[8], a[9], a[10], a[11], a[14]) == (q.at, 256, 4, k.at, 128, 1)
    assert a[15:] == (cos.at, sin.at, 32, 100, q_out.at, STREAM)


def test_tensors_of_another_device_than_the_current_one(calls):
    """The library launches on the current device: tensors of another are refused, on its own default stream too."""
    there = lambda *shape, dtype=F32: Fake(*shape, dtype=dtype, device=1)  # noqa: E731
    table, pos, out = there(1, 4, dtype=I32), there(1, 2, dtype=I32), there(1, 2, 4, 64, dtype=BF16)
    one = lambda dtype=F32: there(2, dtype=dtype)  # noqa: E731
    for stream in (STREAM, 0):
        for call in (lambda: vbq.vbq_kv_append(cache(1), table, pos, there(1, 2, 2, 64), there(1, 2, 2, 64), stream=stream),
                     lambda: vbq.vbq_kv_read(cache(1), table, pos, k_out=there(1, 2, 2, 64), v_out=False, stream=stream),
                     lambda: vbq.vbq_kv_attend(cache(1), table, pos, there(1, 2, 4, 64, dtype=BF16), out=out, workspace=there(4096), stream=stream),
                     lambda: vbq.vbq_residual_norm(there(3, 64), None, there(64), 1e-5, out=there(3, 64, dtype=BF16), stream=stream),
                     lambda: vbq.vbq_sample(there(2, 100), one(), one(I32), one(), one(), one(), tokens=one(I32), probs=False, kept=False,
                                            stream=stream)):
            with pytest.raises(ValueError, match="cuda:1.*cuda:0"):
                call()
    assert calls == []


def test_the_module_is_this_interpreter_s(calls):
    """Its file carries the interpreter's tag, so another Python does not load it and builds its own."""
    import sysconfig
    from paper_2607_02893_gb300 import _decode, build
    assert _decode.__file__ == build.MODULE and build.MODULE.endswith("_decode" + sysconfig.get_config_var("EXT_SUFFIX"))
    assert sysconfig.get_config_var("SOABI") in build.MODULE
