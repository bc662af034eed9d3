"""The causal convolution over as many rows as a call may have."""

import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import delta_oracle as o

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


@pytest.mark.parametrize("rows", [2 ** 31 - 1, 2 ** 31 - 32, 2 ** 31 - 33], ids=["most", "a_tile_less", "and_a_row"])
def test_conv_of_the_most_rows(rows):
    """Row numbers up to 2^31 - 1, with and without starts: rows at both ends and where 32-bit sums of rows and tiles turn
    over, the carried inputs, bit for bit what a short call over the same rows gives."""
    channels, taps = 8, 4
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 80 GB")
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(rows, channels, dtype=torch.bfloat16, device="cuda")
    block = torch.randn(1 << 20, channels, generator=gen, device="cuda").to(torch.bfloat16)
    for at in range(0, rows, 1 << 20):
        x[at:at + (1 << 20)] = block[:rows - at]
    w = torch.randn(channels, taps, generator=gen, device="cuda")
    first = torch.randn(1, taps - 1, channels, generator=gen, device="cuda")
    out = torch.empty(rows, channels, dtype=torch.bfloat16, device="cuda")
    starts = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    for seq in (vbq.Sequences(1, rows), vbq.Sequences(1, rows, starts=starts, tokens=rows)):
        out.fill_(7.0)
        state = first.clone()
        vbq.vbq_causal_conv(seq, x, w, state, out=out)
        assert torch.equal(state[0], x[-3:].float())
        past = first
        for lo in (0, rows // 2, rows - 100):
            part = x[lo:lo + 100].double().cpu().numpy()
            if lo:
                past = x[lo - 3:lo].float()[None]
            y, _, spread = o.causal_conv(part, w.double().cpu().numpy(), past[0].double().cpu().numpy())
            assert o.causal_conv_within_bound(out[lo:lo + 100].double().cpu().numpy(), y, spread).all()
            short = vbq.vbq_causal_conv(vbq.Sequences(1, 100), x[lo:lo + 100].contiguous(), w, past.clone())
            assert torch.equal(out[lo:lo + 100], short)
    assert vbq.vbq_device_status() is None
    del x, out, block
    torch.cuda.empty_cache()
