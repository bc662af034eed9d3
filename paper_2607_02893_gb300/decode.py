"""Binding of the decode step's other operators (include/vbq.h): the 4-bit
key-value cache and its attention, the residual norm, the sampler.

Argument marshalling only, as in vbq.py. Tensors are checked for what the C
call cannot see (type, shape, strides, device); everything else is checked there.
"""

from __future__ import annotations

import ctypes

import torch

from . import vbq as _b
from .vbq import _check

_bf16, _i16, _f32, _i32 = torch.bfloat16, torch.int16, torch.float32, torch.int32
_BF16 = (_bf16, _i16)


class _CacheStruct(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int)]


def _lib():
    return _b._lib or _b.load()


# A decode step makes these calls every few microseconds, so the checks below
# are the few cheapest ones that keep a wrong tensor away from the kernels, and
# the stream is asked for without building a torch.cuda.Stream.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _stream(stream, dev):
    if stream is None:
        return _raw_stream(dev)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _device(t) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError("tensors must be on a GPU")
    return dev


def _type(t) -> int:
    d = t.dtype
    if d is _f32:
        return 1
    if d in _BF16:
        return 0
    raise ValueError(f"expected float32 or bfloat16, got {d}")


def _dense(t, dtype, n, dev, name):
    """Address of a contiguous tensor of n elements of that type on that device."""
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        if dtype is _bf16 and t.dtype is _i16:                  # BF16 bit patterns
            return _dense(t, _i16, n, dev, name)
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on cuda:{dev}, got {t.dtype} "
                         f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")
    return t.data_ptr()


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
        self._as_parameter_ = ctypes.c_void_p(ctypes.addressof(self._struct))


def _rows(cache, table, pos):
    """(device, table, stride, pages, pos, batch, rows) of a cache call."""
    shape, stride = table.shape, table.stride()
    if table.dtype is not _i32 or len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("table must be an int32 tensor (batch, pages) with dense rows")
    pshape = pos.shape
    if pos.dtype is not _i32 or len(pshape) != 2 or not pos.is_contiguous() or pshape[0] != shape[0]:
        raise ValueError("pos must be a contiguous int32 tensor (batch, rows)")
    dev = _device(table)
    if pos.get_device() != dev or cache.device != dev:
        raise ValueError("table, pos and the cache must be on one GPU")
    return dev, table.data_ptr(), stride[0], shape[1], pos.data_ptr(), pshape[0], pshape[1]


def _row_stride(t, b, r, heads, d, dev, name):
    """Elements between rows of a (batch, rows, heads, d) tensor whose rows are dense and evenly spaced."""
    if t.shape != (b, r, heads, d) or t.get_device() != dev:
        raise ValueError(f"{name} must have shape {(b, r, heads, d)} on cuda:{dev}, got {tuple(t.shape)} on {t.device}")
    s0, s1, s2, s3 = t.stride()
    if s3 != 1 or (heads > 1 and s2 != d) or (r > 1 and b > 1 and s0 != r * s1):
        raise ValueError(f"{name}'s rows must be dense and evenly spaced, got strides {t.stride()}")
    return s1 if r > 1 else s0


def vbq_kv_append(cache: KvCache, table, pos, k, v, q=None, cos=None, sin=None, q_out=None, stream=None):
    """Rotate (cos, sin: positions x rot_dim / 2 float32, or None), quantise and
    write the keys and values (batch, rows, kv_heads, head_dim; float32 or
    bfloat16; rows may be slices of a fused product's output) of the tokens at
    pos (batch, rows; negative: unused). With q (batch, rows, heads, head_dim)
    the rotated q is returned as bfloat16 (q_out, allocated when not given)."""
    dev, tp, ts, tn, pp, b, r = _rows(cache, table, pos)
    hk, d = cache.kv_heads, cache.head_dim
    ty = _type(k)
    if v.dtype is not k.dtype or (q is not None and q.dtype is not k.dtype):
        raise ValueError("q, k and v must have one type")
    ks, vs = _row_stride(k, b, r, hk, d, dev, "k"), _row_stride(v, b, r, hk, d, dev, "v")
    qp = op = None
    qs = heads = 0
    if q is not None:
        heads = q.shape[2]
        qs = _row_stride(q, b, r, heads, d, dev, "q")
        if q_out is None:
            q_out = torch.empty((b, r, heads, d), dtype=_bf16, device=q.device)
        qp, op = q.data_ptr(), _dense(q_out, _bf16, b * r * heads * d, dev, "q_out")
    cp = sp = None
    rot = rot_rows = 0
    if cos is not None:
        rot_rows, half = cos.shape
        rot = 2 * half
        cp = _dense(cos, _f32, rot_rows * half, dev, "cos")
        sp = _dense(sin, _f32, rot_rows * half, dev, "sin")
    st = _lib().vbq_kv_append(cache._as_parameter_, tp, ts, tn, pp, b, r, qp, qs, heads, k.data_ptr(), ks, v.data_ptr(), vs,
                              ty, cp, sp, rot, rot_rows, op, _stream(stream, dev))
    if st:
        _check(st)
    return q_out


def vbq_kv_read(cache: KvCache, table, pos, k_out=None, v_out=None, stream=None):
    """What the cache holds for the rows at pos, as float32 (batch, rows,
    kv_heads, head_dim); returns (k_out, v_out), allocating those not given
    (pass False to skip one)."""
    dev, tp, ts, tn, pp, b, r = _rows(cache, table, pos)
    n = b * r * cache.kv_heads * cache.head_dim
    kp = vp = None
    if k_out is None:
        k_out = torch.empty((b, r, cache.kv_heads, cache.head_dim), dtype=_f32, device=pos.device)
    if v_out is None:
        v_out = torch.empty((b, r, cache.kv_heads, cache.head_dim), dtype=_f32, device=pos.device)
    if k_out is not False:
        kp = _dense(k_out, _f32, n, dev, "k_out")
    if v_out is not False:
        vp = _dense(v_out, _f32, n, dev, "v_out")
    st = _lib().vbq_kv_read(cache._as_parameter_, tp, ts, tn, pp, b, r, kp, vp, _stream(stream, dev))
    if st:
        _check(st)
    return None if k_out is False else k_out, None if v_out is False else v_out


def vbq_kv_workspace_bytes(cache: KvCache, batch: int, rows: int, heads: int) -> int:
    out = ctypes.c_size_t()
    _check(_lib().vbq_kv_workspace_bytes(cache, int(batch), int(rows), int(heads), ctypes.byref(out)))
    return out.value


def vbq_kv_workspace(cache: KvCache, batch: int, rows: int, heads: int):
    """A zeroed workspace for vbq_kv_attend calls that need no more than these sizes do."""
    n = vbq_kv_workspace_bytes(cache, batch, rows, heads)
    return torch.zeros(n, dtype=torch.uint8, device=cache.pages.device)


def vbq_kv_attend(cache: KvCache, table, pos, q, scale=None, window: int = 0, out=None, workspace=None, stream=None):
    """Attention of q (batch, rows, heads, head_dim bfloat16) over the cache, each
    row over the keys in (pos - window, pos] of its sequence (window 0: all).
    scale defaults to head_dim ** -0.5. Returns out (bfloat16, as q). Give the
    workspace of vbq_kv_workspace to keep it between calls; one is made (and
    zeroed) for this call otherwise."""
    dev, tp, ts, tn, pp, b, r = _rows(cache, table, pos)
    heads, d = q.shape[2], cache.head_dim
    n = b * r * heads * d
    if q.dim() != 4 or q.shape[3] != d:
        raise ValueError(f"q must have shape {(b, r, 'heads', d)}, got {tuple(q.shape)}")
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = vbq_kv_workspace(cache, b, r, heads)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the cache's GPU")
    st = _lib().vbq_kv_attend(cache._as_parameter_, tp, ts, tn, pp, b, r, _dense(q, _bf16, n, dev, "q"), heads,
                              d ** -0.5 if scale is None else scale, window, _dense(out, _bf16, n, dev, "out"),
                              workspace.data_ptr(), workspace.nbytes, _stream(stream, dev))
    if st:
        _check(st)
    return out


def vbq_residual_norm(x, residual, weight, eps: float, out=None, residual_out=None, stream=None):
    """r' = residual + x in the residual's type (x itself when residual is None)
    and out = r' * rsqrt(mean(r'^2) + eps) * weight as bfloat16, per row of the
    last dimension. Returns (out, residual_out), allocating those not given;
    residual_out may be residual itself."""
    dev, n, xt = _device(x), x.numel(), _type(x)
    width = x.shape[-1]
    if out is None:
        out = torch.empty(x.shape, dtype=_bf16, device=x.device)
    rp = ro = None
    rt = 0
    if residual is not None:
        rt, rd = _type(residual), residual.dtype
        if residual_out is None:
            residual_out = torch.empty_like(residual)
        rp = _dense(residual, rd, n, dev, "residual")
        ro = rp if residual_out is residual else _dense(residual_out, rd, n, dev, "residual_out")
    st = _lib().vbq_residual_norm(_dense(x, x.dtype, n, dev, "x"), xt, rp, rt, _dense(weight, _f32, width, dev, "weight"),
                                  eps, n // width if width else 0, width, _dense(out, _bf16, n, dev, "out"), ro,
                                  _stream(stream, dev))
    if st:
        _check(st)
    return out, residual_out


def vbq_sample(logits, temperature, top_k, top_p, min_p, u, tokens=None, probs=None, kept=None, stream=None):
    """Draw one token per row of logits (batch, vocab; float32 or bfloat16) under
    per-row temperature, top_p, min_p, u (float32) and top_k (int32), all of
    shape (batch,). Returns (tokens, probs, kept), allocating those not given
    (pass False to skip probs or kept)."""
    dev = _device(logits)
    b, vocab = logits.shape
    stride, unit = logits.stride()
    if unit != 1 and vocab > 1:
        raise ValueError("logits' rows must be dense")
    if tokens is None:
        tokens = torch.empty(b, dtype=_i32, device=logits.device)
    if probs is None:
        probs = torch.empty(b, dtype=_f32, device=logits.device)
    if kept is None:
        kept = torch.empty(b, dtype=_i32, device=logits.device)
    st = _lib().vbq_sample(logits.data_ptr(), stride, _type(logits), b, vocab,
                           _dense(temperature, _f32, b, dev, "temperature"), _dense(top_k, _i32, b, dev, "top_k"),
                           _dense(top_p, _f32, b, dev, "top_p"), _dense(min_p, _f32, b, dev, "min_p"),
                           _dense(u, _f32, b, dev, "u"), _dense(tokens, _i32, b, dev, "tokens"),
                           None if probs is False else _dense(probs, _f32, b, dev, "probs"),
                           None if kept is False else _dense(kept, _i32, b, dev, "kept"), _stream(stream, dev))
    if st:
        _check(st)
    return tokens, None if probs is False else probs, None if kept is False else kept
