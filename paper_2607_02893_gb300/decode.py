"""Binding of the decode step's other operators (include/vbq.h): the 4-bit
key-value cache and its attention, the residual norm, the sampler.

Argument marshalling only, as in vbq.py. Tensors are checked for what the C
call cannot see (type, shape, strides, device); everything else is checked there.
"""

from __future__ import annotations

import ctypes

import torch

from . import vbq as _b
from .vbq import _check, _stream

_BF16 = (torch.bfloat16, torch.int16)


class _CacheStruct(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int)]


def _lib():
    return _b._lib or _b.load()


def _type(t) -> int:
    if t.dtype is torch.float32:
        return 1
    if t.dtype in _BF16:
        return 0
    raise ValueError(f"expected float32 or bfloat16, got {t.dtype}")


def _dense(t, dtypes, shape, name):
    """Address of a contiguous tensor of that type and shape."""
    if t.dtype not in dtypes or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtypes[0]} tensor of shape {shape}, got "
                         f"{t.dtype} {tuple(t.shape)} with strides {t.stride()}")
    return t.data_ptr()


_I32 = (torch.int32,)
_F32 = (torch.float32,)


def _same_device(first, *rest):
    if not first.is_cuda:
        raise ValueError("tensors must be on a GPU")
    for t in rest:
        if t is not None and t.device != first.device:
            raise ValueError(f"tensors on {first.device} and {t.device}")


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
        self._struct = _CacheStruct(pages.data_ptr(), self.n_pages, self.kv_heads, self.head_dim)
        self._as_parameter_ = ctypes.c_void_p(ctypes.addressof(self._struct))


def _rows(cache, table, pos):
    """(table, stride, pages, pos, batch, rows) of a cache call."""
    if table.dtype is not torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be an int32 tensor (batch, pages) with dense rows")
    if pos.dtype is not torch.int32 or pos.dim() != 2 or not pos.is_contiguous() or pos.shape[0] != table.shape[0]:
        raise ValueError("pos must be a contiguous int32 tensor (batch, rows)")
    _same_device(cache.pages, table, pos)
    b, r = pos.shape
    return table.data_ptr(), table.stride(0), table.shape[1], pos.data_ptr(), b, r


def _row_stride(t, b, r, heads, d, name):
    """Elements between rows of a (batch, rows, heads, d) tensor whose rows are dense and evenly spaced."""
    if t.dim() != 4 or t.shape[0] != b or t.shape[1] != r or t.shape[2] != heads or t.shape[3] != d:
        raise ValueError(f"{name} must have shape {(b, r, heads, d)}, got {tuple(t.shape)}")
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
    tp, ts, tn, pp, b, r = _rows(cache, table, pos)
    hk, d = cache.kv_heads, cache.head_dim
    ty = _type(k)
    if v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise ValueError("q, k and v must have one type")
    ks, vs = _row_stride(k, b, r, hk, d, "k"), _row_stride(v, b, r, hk, d, "v")
    qp = op = None
    qs = heads = 0
    if q is not None:
        heads = q.shape[2]
        qs = _row_stride(q, b, r, heads, d, "q")
        if q_out is None:
            q_out = torch.empty((b, r, heads, d), dtype=torch.bfloat16, device=q.device)
        qp, op = q.data_ptr(), _dense(q_out, _BF16, (b, r, heads, d), "q_out")
    cp = sp = None
    rot = rot_rows = 0
    if cos is not None:
        rot_rows, rot = cos.shape[0], 2 * cos.shape[1]
        cp = _dense(cos, _F32, (rot_rows, rot // 2), "cos")
        sp = _dense(sin, _F32, (rot_rows, rot // 2), "sin")
    _same_device(cache.pages, k, v, q, q_out, cos, sin)
    _check(_lib().vbq_kv_append(cache, tp, ts, tn, pp, b, r, qp, qs, heads, k.data_ptr(), ks, v.data_ptr(), vs, ty,
                                cp, sp, rot, rot_rows, op, _stream(stream, k)))
    return q_out


def vbq_kv_read(cache: KvCache, table, pos, k_out=None, v_out=None, stream=None):
    """What the cache holds for the rows at pos, as float32 (batch, rows,
    kv_heads, head_dim); returns (k_out, v_out), allocating those not given
    (pass False to skip one)."""
    tp, ts, tn, pp, b, r = _rows(cache, table, pos)
    shape = (b, r, cache.kv_heads, cache.head_dim)
    k_out, v_out = (torch.empty(shape, dtype=torch.float32, device=pos.device) if o is None else o if o is not False else None
                    for o in (k_out, v_out))
    ptrs = [None if o is None else _dense(o, _F32, shape, "k_out and v_out") for o in (k_out, v_out)]
    _same_device(cache.pages, k_out, v_out)
    _check(_lib().vbq_kv_read(cache, tp, ts, tn, pp, b, r, ptrs[0], ptrs[1], _stream(stream, pos)))
    return k_out, v_out


def vbq_kv_workspace_bytes(cache: KvCache, batch: int, rows: int, heads: int) -> int:
    out = ctypes.c_size_t()
    _check(_lib().vbq_kv_workspace_bytes(cache, int(batch), int(rows), int(heads), ctypes.byref(out)))
    return out.value


def vbq_kv_workspace(cache: KvCache, batch: int, rows: int, heads: int):
    """A zeroed workspace for vbq_kv_attend calls of at most these sizes."""
    n = vbq_kv_workspace_bytes(cache, batch, rows, heads)
    return torch.zeros(n, dtype=torch.uint8, device=cache.pages.device)


def vbq_kv_attend(cache: KvCache, table, pos, q, scale=None, window: int = 0, out=None, workspace=None, stream=None):
    """Attention of q (batch, rows, heads, head_dim bfloat16) over the cache, each
    row over the keys in (pos - window, pos] of its sequence (window 0: all).
    scale defaults to head_dim ** -0.5. Returns out (bfloat16, as q). Give the
    workspace of vbq_kv_workspace to keep it between calls; one is made (and
    zeroed) for this call otherwise."""
    tp, ts, tn, pp, b, r = _rows(cache, table, pos)
    heads, d = q.shape[2], cache.head_dim
    qp = _dense(q, _BF16, (b, r, heads, d), "q")
    if out is None:
        out = torch.empty_like(q)
    op = _dense(out, _BF16, (b, r, heads, d), "out")
    if workspace is None:
        workspace = vbq_kv_workspace(cache, b, r, heads)
    _same_device(cache.pages, q, out, workspace)
    _check(_lib().vbq_kv_attend(cache, tp, ts, tn, pp, b, r, qp, heads, d ** -0.5 if scale is None else scale, window,
                                op, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                _stream(stream, q)))
    return out


def vbq_residual_norm(x, residual, weight, eps: float, out=None, residual_out=None, stream=None):
    """r' = residual + x in the residual's type (x itself when residual is None)
    and out = r' * rsqrt(mean(r'^2) + eps) * weight as bfloat16, per row of the
    last dimension. Returns (out, residual_out), allocating those not given;
    residual_out may be residual itself."""
    shape = tuple(x.shape)
    width = shape[-1]
    rows = x.numel() // width if width else 0
    if out is None:
        out = torch.empty(shape, dtype=torch.bfloat16, device=x.device)
    rp = ro = None
    rt = 0
    if residual is not None:
        rt = _type(residual)
        if residual_out is None:
            residual_out = torch.empty_like(residual)
        rp = _dense(residual, (residual.dtype,), shape, "residual")
        ro = _dense(residual_out, (residual.dtype,), shape, "residual_out")
    _same_device(x, residual, weight, out, residual_out)
    _check(_lib().vbq_residual_norm(_dense(x, (x.dtype,), shape, "x"), _type(x), rp, rt,
                                    _dense(weight, _F32, (width,), "weight"), eps, rows, width,
                                    _dense(out, _BF16, shape, "out"), ro, _stream(stream, x)))
    return out, residual_out


def vbq_sample(logits, temperature, top_k, top_p, min_p, u, tokens=None, probs=None, kept=None, stream=None):
    """Draw one token per row of logits (batch, vocab; float32 or bfloat16) under
    per-row temperature, top_p, min_p, u (float32) and top_k (int32), all of
    shape (batch,). Returns (tokens, probs, kept), allocating those not given
    (pass False to skip probs or kept)."""
    b, vocab = logits.shape
    if vocab > 1 and logits.stride(1) != 1:
        raise ValueError("logits' rows must be dense")
    n, dev = (b,), logits.device
    if tokens is None:
        tokens = torch.empty(n, dtype=torch.int32, device=dev)
    probs = torch.empty(n, dtype=torch.float32, device=dev) if probs is None else probs if probs is not False else None
    kept = torch.empty(n, dtype=torch.int32, device=dev) if kept is None else kept if kept is not False else None
    _same_device(logits, temperature, top_k, top_p, min_p, u, tokens, probs, kept)
    _check(_lib().vbq_sample(logits.data_ptr(), logits.stride(0), _type(logits), b, vocab,
                             _dense(temperature, _F32, n, "temperature"), _dense(top_k, _I32, n, "top_k"),
                             _dense(top_p, _F32, n, "top_p"), _dense(min_p, _F32, n, "min_p"), _dense(u, _F32, n, "u"),
                             _dense(tokens, _I32, n, "tokens"), None if probs is None else _dense(probs, _F32, n, "probs"),
                             None if kept is None else _dense(kept, _I32, n, "kept"), _stream(stream, logits)))
    return tokens, probs, kept
