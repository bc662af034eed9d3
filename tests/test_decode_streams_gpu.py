"""Decode calls on a stream of their own, while the current stream is busy before
and after them: nothing that a call makes for itself may be reached by the
current stream's work."""

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


@pytest.mark.parametrize("form", ["object", "handle"])
def test_calls_on_another_stream_without_workspace_or_outputs(form):
    torch.manual_seed(1)
    hk, heads, d, n = 2, 8, 128, 9000
    pages = -(-n // 64)
    cache = vbq.KvCache(pages, hk, d)
    table = torch.randperm(pages, device=DEV).to(I32)[None].contiguous()
    k, v = (torch.randn(1, n, hk, d, device=DEV).to(torch.bfloat16) for _ in "kv")
    vbq.vbq_kv_append(cache, table, torch.arange(n, dtype=I32, device=DEV)[None], k, v)
    pos = torch.tensor([[n - 1]], dtype=I32, device=DEV)
    q = torch.randn(1, 1, heads, d, device=DEV).to(torch.bfloat16)
    x, w = torch.randn(40, 4096, device=DEV), torch.rand(4096, device=DEV)
    logits = torch.randn(3, 128256, device=DEV)
    one = lambda a, t=torch.float32: torch.full((3,), a, dtype=t, device=DEV)  # noqa: E731
    params = (one(1.0), one(50, I32), one(0.9), one(0.0), one(0.4))

    def calls(stream=None):
        return [vbq.vbq_kv_attend(cache, table, pos, q, stream=stream), *vbq.vbq_residual_norm(x, x, w, 1e-5, stream=stream),
                *vbq.vbq_sample(logits, *params, stream=stream), *vbq.vbq_kv_read(cache, table, pos, stream=stream),
                vbq.vbq_kv_append(cache, table, pos, k[:, -1:], v[:, -1:], q=q, stream=stream)]

    want = [t.clone() for t in calls()]
    side = torch.cuda.Stream()
    stream = side if form == "object" else side.cuda_stream
    size = vbq.vbq_kv_workspace_bytes(cache, 1, 1, heads)
    big = torch.randn(8192, 8192, device=DEV)
    torch.cuda.synchronize()
    for _ in range(10):
        junk = [torch.full((size,), 0xff, dtype=torch.uint8, device=DEV) for _ in range(3)]      # the current stream's pool: not zeros
        del junk
        for _ in range(4):
            torch.mm(big, big)                                    # some milliseconds: zeros on this stream would come late
        got = calls(stream)
        junk = [torch.full((size,), 0xff, dtype=torch.uint8, device=DEV) for _ in range(3)]
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        del junk, got
    assert vbq.vbq_device_status() is None
