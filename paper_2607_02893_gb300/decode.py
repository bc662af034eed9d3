"""Binding of the decode step's other operators (include/vbq.h): the 4-bit
key-value cache and its attention, the residual norm, the sampler.

Argument marshalling only, as in vbq.py. A decode step makes these calls every
few microseconds, so their checks (of what the C call cannot see: a tensor's
type, size, strides and device, which has to be the current one) and the calls
themselves are in the CPython module native/_decode.c, built beside libvbq.so;
the ones that are not in a step's way go through ctypes.

Outputs and a workspace that a call is not given are made on the stream that the
call is enqueued on (`stream`, or PyTorch's current one), as by a caller under
torch.cuda.stream(stream): the allocator then keeps their memory in that stream's
order, and zeros are there before the kernel that needs them.
"""

from __future__ import annotations

import contextlib
import ctypes

import torch

from . import vbq as _b
from .vbq import _check

_native = None


def _load():
    """The marshalling module, given the library's entry points. Fails loudly if absent."""
    global _native
    lib = _b.load()
    try:
        from . import _decode
    except ImportError as e:
        from .build import MODULE
        raise RuntimeError(f"VBQ decode binding not built: {MODULE} ({e}); "
                           "run `python -c 'import __graft_entry__ as g; g.build()'`") from e
    raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    current_device = None                                         # asked (0.3 us a call) where there is another one
    if torch.cuda.device_count() > 1:
        current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
    _decode.setup(torch.float32, torch.bfloat16, torch.int16, torch.int32, raw_stream, current_device,
                  address(lib.vbq_kv_append), address(lib.vbq_kv_read), address(lib.vbq_kv_attend),
                  address(lib.vbq_residual_norm), address(lib.vbq_sample))
    _native = _decode
    return _decode


def _lib():
    return _b._lib or _b.load()


def _on(stream, device):
    """The context in which to make a call's tensors."""
    if stream is None or device.type != "cuda":
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        handle = stream if isinstance(stream, int) else stream.cuda_stream
        # 0 and 1 (cudaStreamLegacy) are the default stream
        stream = torch.cuda.default_stream(device) if handle in (0, 1) else torch.cuda.ExternalStream(handle, device=device)
    return torch.cuda.stream(stream)


class _CacheStruct(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int)]


def vbq_kv_page_bytes(kv_heads: int, head_dim: int) -> int:
    """Bytes of one page (64 tokens of every key-value head)."""
    out = ctypes.c_size_t()
    _check(_lib().vbq_kv_page_bytes(int(kv_heads), int(head_dim), ctypes.byref(out)))
    return out.value


class KvCache:
    """A 4-bit key-value cache of n_pages pages of 64 tokens. Owns its device
    memory as a torch tensor (`pages`, uint8), or takes the caller's."""

    def __init__(self, n_pages: int, kv_heads: int, head_dim: int, device="cuda", pages=None):
        per = vbq_kv_page_bytes(kv_heads, head_dim)
        if pages is None:
            pages = torch.empty(int(n_pages) * per, dtype=torch.uint8, device=device)
        elif pages.dtype != torch.uint8 or not pages.is_contiguous() or pages.numel() < int(n_pages) * per:
            raise ValueError(f"pages must be a contiguous uint8 tensor of at least {int(n_pages) * per} bytes")
        self.pages = pages
        self.n_pages, self.kv_heads, self.head_dim = int(n_pages), int(kv_heads), int(head_dim)
        self.device = pages.get_device()
        self._struct = _CacheStruct(pages.data_ptr(), self.n_pages, self.kv_heads, self.head_dim)
        self._address = ctypes.addressof(self._struct)
        self._as_parameter_ = ctypes.c_void_p(self._address)


def vbq_kv_append(cache: KvCache, table, pos, k, v, q=None, cos=None, sin=None, q_out=None, stream=None):
    """Rotate (cos, sin: positions x rot_dim / 2 float32, or None), quantise and
    write the keys and values (batch, rows, kv_heads, head_dim; float32 or
    bfloat16; rows may be slices of a fused product's output) of the tokens at
    pos (batch, rows; negative: unused). With q (batch, rows, heads, head_dim)
    the rotated q is returned as bfloat16 (q_out, allocated when not given)."""
    if q is not None and q_out is None:
        with _on(stream, q.device):
            q_out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    st = (_native or _load()).append(cache._address, cache.device, table, pos, k, v, q, cos, sin, q_out, stream)
    if st:
        _check(st)
    return q_out


def vbq_kv_read(cache: KvCache, table, pos, k_out=None, v_out=None, stream=None):
    """What the cache holds for the rows at pos, as float32 (batch, rows,
    kv_heads, head_dim); returns (k_out, v_out), allocating those not given
    (pass False to skip one)."""
    if k_out is None or v_out is None:
        shape = (*pos.shape, cache.kv_heads, cache.head_dim)
        with _on(stream, pos.device):
            k_out = torch.empty(shape, dtype=torch.float32, device=pos.device) if k_out is None else k_out
            v_out = torch.empty(shape, dtype=torch.float32, device=pos.device) if v_out is None else v_out
    st = (_native or _load()).read(cache._address, cache.device, table, pos, k_out, v_out, stream)
    if st:
        _check(st)
    return None if k_out is False else k_out, None if v_out is False else v_out


def vbq_kv_workspace_bytes(cache: KvCache, batch: int, rows: int, heads: int) -> int:
    out = ctypes.c_size_t()
    _check(_lib().vbq_kv_workspace_bytes(cache, int(batch), int(rows), int(heads), ctypes.byref(out)))
    return out.value


def vbq_kv_workspace(cache: KvCache, batch: int, rows: int, heads: int, stream=None):
    """A workspace for vbq_kv_attend calls that need no more than these sizes do,
    zeroed on `stream` (PyTorch's current one by default): calls on another wait for that first."""
    n = vbq_kv_workspace_bytes(cache, batch, rows, heads)
    with _on(stream, cache.pages.device):
        return torch.zeros(n, dtype=torch.uint8, device=cache.pages.device)


def vbq_kv_attend(cache: KvCache, table, pos, q, scale=None, window: int = 0, out=None, workspace=None, stream=None):
    """Attention of q (batch, rows, heads, head_dim bfloat16) over the cache, each
    row over the keys in (pos - window, pos] of its sequence (window 0: all).
    scale defaults to head_dim ** -0.5. Returns out (bfloat16, as q). Give the
    workspace of vbq_kv_workspace to keep it between calls; one is made (and
    zeroed) for this call otherwise."""
    if out is None:
        with _on(stream, q.device):
            out = torch.empty_like(q)
    if workspace is None:
        workspace = vbq_kv_workspace(cache, q.shape[0], q.shape[1], q.shape[2], stream)
    st = (_native or _load()).attend(cache._address, cache.device, table, pos, q, scale, window, out, workspace, stream)
    if st:
        _check(st)
    return out


def vbq_residual_norm(x, residual, weight, eps: float, out=None, residual_out=None, stream=None):
    """r' = residual + x in the residual's type (x itself when residual is None)
    and out = r' * rsqrt(mean(r'^2) + eps) * weight as bfloat16, per row of the
    last dimension. Returns (out, residual_out), allocating those not given;
    residual_out may be residual itself."""
    if out is None or (residual is not None and residual_out is None):
        with _on(stream, x.device):
            out = torch.empty(x.shape, dtype=torch.bfloat16, device=x.device) if out is None else out
            residual_out = torch.empty_like(residual) if residual is not None and residual_out is None else residual_out
    st = (_native or _load()).norm(x, residual, weight, eps, out, residual_out, stream)
    if st:
        _check(st)
    return out, residual_out


def vbq_sample(logits, temperature, top_k, top_p, min_p, u, tokens=None, probs=None, kept=None, stream=None):
    """Draw one token per row of logits (batch, vocab; float32 or bfloat16) under
    per-row temperature, top_p, min_p, u (float32) and top_k (int32), all of
    shape (batch,). Returns (tokens, probs, kept), allocating those not given
    (pass False to skip probs or kept)."""
    b, dev = logits.shape[0], logits.device
    if tokens is None or probs is None or kept is None:
        with _on(stream, dev):
            tokens = torch.empty(b, dtype=torch.int32, device=dev) if tokens is None else tokens
            probs = torch.empty(b, dtype=torch.float32, device=dev) if probs is None else probs
            kept = torch.empty(b, dtype=torch.int32, device=dev) if kept is None else kept
    st = (_native or _load()).sample(logits, temperature, top_k, top_p, min_p, u, tokens, probs, kept, stream)
    if st:
        _check(st)
    return tokens, None if probs is False else probs, None if kept is False else kept
