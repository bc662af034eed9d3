"""Tensors that a decode call makes for itself belong to the stream it is
enqueued on. CPU only: torch's allocations and streams are stood in for, and
nothing is launched."""

import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2607_02893_gb300 import decode

DEV = SimpleNamespace(type="cuda", index=0)


def fake(*shape):
    return SimpleNamespace(shape=shape, device=DEV, dtype=torch.bfloat16)


@pytest.fixture
def made(monkeypatch):
    """The streams under which tensors were made, one per tensor, and the calls' streams."""
    log = SimpleNamespace(on=[], calls=[])
    current = [None]

    @contextlib.contextmanager
    def under(stream):
        before, current[0] = current[0], stream
        yield
        current[0] = before

    def make(like, *a, **k):
        log.on.append(current[0])
        return fake(*(getattr(like, "shape", None) or (like,)))

    for name in ("empty", "empty_like", "zeros"):
        monkeypatch.setattr(torch, name, make)
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: 0)
    call = lambda *a: log.calls.append(a[-1]) or 0  # noqa: E731
    monkeypatch.setattr(decode, "_native", SimpleNamespace(append=call, read=call, attend=call, norm=call, sample=call))
    monkeypatch.setattr(decode, "vbq_kv_workspace_bytes", lambda *a: 1024)
    return log


CACHE = SimpleNamespace(_address=0, device=0, kv_heads=2, head_dim=64, pages=SimpleNamespace(device=DEV))

CALLS = {
    "append": (lambda s: decode.vbq_kv_append(CACHE, fake(1, 1), fake(1, 1), fake(1, 1, 2, 64), fake(1, 1, 2, 64), q=fake(1, 1, 4, 64), stream=s), 1),
    "read": (lambda s: decode.vbq_kv_read(CACHE, fake(1, 1), fake(1, 1), stream=s), 2),
    "attend": (lambda s: decode.vbq_kv_attend(CACHE, fake(1, 1), fake(1, 1), fake(1, 1, 4, 64), stream=s), 2),
    "norm": (lambda s: decode.vbq_residual_norm(fake(2, 8), fake(2, 8), fake(8), 1e-5, stream=s), 2),
    "sample": (lambda s: decode.vbq_sample(fake(2, 100), *(fake(2) for _ in range(5)), stream=s), 3),
}


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("stream", [4096, SimpleNamespace(cuda_stream=8192)], ids=["handle", "object"])
def test_tensors_are_made_on_the_call_s_stream(made, name, stream):
    call, n = CALLS[name]
    call(stream)
    handle = stream if isinstance(stream, int) else stream.cuda_stream
    assert made.on == [handle] * n and made.calls == [stream]


@pytest.mark.parametrize("name", sorted(CALLS))
def test_tensors_are_made_on_the_current_stream_without_one(made, name):
    call, n = CALLS[name]
    call(None)
    assert made.on == [None] * n and made.calls == [None]


@pytest.mark.parametrize("handle", [0, 1])
def test_handles_of_the_default_stream(made, handle):
    CALLS["attend"][0](handle)
    assert made.on == [0, 0] and made.calls == [handle]


def test_workspace_takes_a_stream(made):
    decode.vbq_kv_workspace(CACHE, 1, 1, 4, stream=4096)
    decode.vbq_kv_workspace(CACHE, 1, 1, 4)
    assert made.on == [4096, None]
