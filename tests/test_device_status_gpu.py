"""vbq_device_status and the calls on sequences that report to it."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_first_call_of_a_process_may_be_captured():
    """Nothing that a call on sequences looks up once per device stands in a capture's way; a slot outside the pool is reported
    from the replay."""
    code = """
import torch, paper_2607_02893_gb300 as vbq
d = "cuda"
x, w, state = torch.randn(2, 64, device=d), torch.randn(64, 4, device=d), torch.zeros(1, 3, 64, device=d)
q = torch.randn(2, 1, 64, device=d).to(torch.bfloat16)
gate, s = torch.zeros(2, 1, device=d), torch.zeros(1, 1, 64, 64, device=d)
seq = vbq.Sequences(2, 1)
out, o = torch.empty(2, 64, dtype=torch.bfloat16, device=d), torch.empty_like(q)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    vbq.vbq_causal_conv(seq, x, w, state, out=out)
    vbq.vbq_delta_rule(seq, s, q, q, q, gate, gate + 0.5, out=o)
assert vbq.vbq_device_status() is None
graph.replay()
try:
    vbq.vbq_device_status()
except vbq.VbqError as e:
    assert "pool" in str(e)
else:
    raise AssertionError("not reported")
assert vbq.vbq_device_status() is None and out[0].any() and not out[1].any() and not o[1].any()
print("fine")
"""
    from paper_2607_02893_gb300 import build
    build.build()
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]
