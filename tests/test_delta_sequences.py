"""What a Sequences refuses before any call."""

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
