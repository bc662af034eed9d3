"""Binding of the operators of a linear-attention layer (include/vbq.h): the short
causal convolution, the gated delta rule and the gated norm per head.

As in decode.py: checks of what the C call cannot see and the calls themselves
are in native/_decode.c, outputs that a call is not given are made on the call's
stream, tensors have to be on the current device.
"""

from __future__ import annotations

import ctypes

import torch

from . import decode as _d
from . import vbq as _b
from .decode import _on
from .vbq import _check

_native = None


def _load():
    """The marshalling module, given these operators' entry points."""
    global _native
    native = _d._native or _d._load()
    lib = _b.load()
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
    native.setup_delta(address(lib.vbq_causal_conv), address(lib.vbq_delta_rule), address(lib.vbq_gated_norm))
    _native = native
    return native


class _SequencesStruct(ctypes.Structure):
    _fields_ = [("starts", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("fresh", ctypes.c_void_p), ("batch", ctypes.c_int),
                ("rows", ctypes.c_int), ("tokens", ctypes.c_int64)]


class Sequences:
    """Whose tokens the rows of a call are: `batch` sequences of `rows` rows each, or with starts (batch + 1) sequence b's
    rows starts[b] .. starts[b + 1] - 1 of `tokens` (`rows`: the longest's number). slots (batch): where each sequence's
    state is in its pool (its number without it; negative: unused). fresh (batch): not 0 where a sequence begins. All
    int32 on the GPU, kept here and read by the calls, so their values may change between calls (and between a graph's
    replays); one Sequences serves every layer of a step."""

    def __init__(self, batch: int, rows: int, starts=None, tokens: int | None = None, slots=None, fresh=None):
        batch, rows = int(batch), int(rows)
        if not 0 <= batch < 1 << 31 or not 0 <= rows < 1 << 31:
            raise ValueError("batch and rows must be within 0..2^31 - 1")
        if starts is None:
            if tokens is not None and int(tokens) != batch * rows:
                raise ValueError("without starts, tokens is batch * rows")
            tokens = batch * rows
        elif tokens is None:
            raise ValueError("starts needs tokens, the rows of the calls' arrays")
        tokens = int(tokens)
        if not 0 <= tokens < 1 << 63:
            raise ValueError("tokens must be within 0..2^63 - 1")
        self.batch, self.rows, self.tokens = batch, rows, tokens
        self.starts, self.slots, self.fresh = starts, slots, fresh
        self.device = -1                                          # any
        for name, t, n in (("starts", starts, batch + 1), ("slots", slots, batch), ("fresh", fresh, batch)):
            if t is None:
                continue
            if t.dtype != torch.int32 or t.numel() != n or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int32 tensor of {n} elements")
            if t.get_device() < 0:
                raise ValueError(f"{name} must be on a GPU")
            if self.device >= 0 and t.get_device() != self.device:
                raise ValueError("starts, slots and fresh must be on one GPU")
            self.device = t.get_device()
        at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self._struct = _SequencesStruct(at(starts), at(slots), at(fresh), batch, rows, self.tokens)
        self._address = ctypes.addressof(self._struct)
        self._as_parameter_ = ctypes.c_void_p(self._address)


def vbq_causal_conv(seq: Sequences, x, weight, state, bias=None, silu: bool = True, out=None, stream=None):
    """The causal convolution per channel of x (tokens, channels; float32 or bfloat16; rows may be slices of a product's
    output) with weight (channels, taps), bias (channels) or None, and silu or not. state (n_slots, taps - 1, channels)
    holds each sequence's last inputs, the oldest first, and is moved on. weight, bias and state are float32. Returns out
    (tokens, channels bfloat16)."""
    if out is None:
        with _on(stream, x.device):
            out = torch.empty(x.shape, dtype=torch.bfloat16, device=x.device)
    st = (_native or _load()).conv(seq._address, seq.device, x, weight, bias, state, silu, out, stream)
    if st:
        _check(st)
    return out


def vbq_delta_rule(seq: Sequences, state, q, k, v, decay, beta, a_log=None, dt_bias=None, scale=None, normalize: bool = True,
                   out=None, stream=None):
    """The gated delta rule over q, k (tokens, k_heads, head_k) and v (tokens, heads, head_v), all float32 or all bfloat16,
    whose rows may be slices of wider ones. decay and beta (tokens, heads), both float32 or both bfloat16, are the inputs
    of the gates with a_log and dt_bias (heads, float32), else the log decay and the factor themselves. scale defaults to
    head_k ** -0.5; normalize brings q and k to unit length. state (n_slots, heads, head_k, head_v float32) is moved on.
    Returns out (tokens, heads, head_v bfloat16)."""
    if out is None:
        with _on(stream, v.device):
            out = torch.empty(v.shape, dtype=torch.bfloat16, device=v.device)
    st = (_native or _load()).delta(seq._address, seq.device, state, q, k, v, decay, beta, a_log, dt_bias, scale, normalize, out, stream)
    if st:
        _check(st)
    return out


def vbq_gated_norm(x, gate, weight, eps: float, out=None, stream=None):
    """x * rsqrt(mean(x^2) + eps) * weight * silu(gate) over the last dimension of x (rows, heads, width), as bfloat16. x and
    gate are float32 or bfloat16, each on its own, and their rows may be slices of wider ones; gate may be None."""
    if out is None:
        with _on(stream, x.device):
            out = torch.empty(x.shape, dtype=torch.bfloat16, device=x.device)
    st = (_native or _load()).gated(x, gate, weight, eps, out, stream)
    if st:
        _check(st)
    return out
