"""What a Sequences refuses before any call, and a call of one."""

import ctypes

import pytest
import torch

import paper_2607_02893_gb300 as vbq


class Starts:
    """Stands for an int32 tensor of three elements on a GPU."""
    dtype = torch.int32

    def numel(self):
        return 3

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0

    def data_ptr(self):
        return 1 << 20


@pytest.mark.parametrize("tokens", [-1, 1 << 63, (1 << 64) + 6, -(1 << 64) + 6])
def test_tokens_that_64_bits_do_not_hold(tokens):
    """A count that wrapped around would be taken for another one."""
    with pytest.raises(ValueError, match="tokens"):
        vbq.Sequences(2, 3, starts=Starts(), tokens=tokens)
    assert vbq.Sequences(2, 3, starts=Starts(), tokens=6)._struct.tokens == 6


def test_tokens_of_a_delta_rule():
    """Row numbers are rounded up to a chunk's end in 32 bits."""
    from paper_2607_02893_gb300 import build
    from paper_2607_02893_gb300.delta import _SequencesStruct
    build.build()
    lib = vbq.load()
    buf = ctypes.create_string_buffer(64)
    p = (ctypes.addressof(buf) + 15) // 16 * 16
    for tokens in ((1 << 31) - 63, (1 << 31) - 1):
        seq = _SequencesStruct(p, None, None, 1, 5, tokens)
        assert lib.vbq_delta_rule(ctypes.byref(seq), p, 1, p, 64, p, 64, p, 64, 1, 1, 64, 1, 64, p, 1, p, 1, 0, None, None, 1.0, 1, p, None) == -7
        assert "2^31 - 64" in lib.vbq_last_error().decode()
