"""CPU oracle of a linear-attention layer's operators, plain numpy in fp64: the
causal convolution, the gated delta rule token by token, the gated norm. Written
from the definitions in include/vbq.h; it shares no code with the CUDA path."""

from __future__ import annotations

import numpy as np

UNIT_EPS = 1e-6
CHUNK = 64


def silu(x):
    with np.errstate(over="ignore"):
        return x / (1.0 + np.exp(-x))


def causal_conv(x, weight, carried, bias=None, act=True):
    """One sequence: x (rows, channels), weight (channels, taps), carried (taps - 1, channels). Returns (y, the inputs
    carried on, spread): spread is the sum of |w x| and |bias| per output, for the error bound."""
    x, weight = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    taps = weight.shape[1]
    line = np.concatenate((np.asarray(carried, np.float64), x), 0)
    y = sum(line[j:j + len(x)] * weight[:, j] for j in range(taps))
    spread = sum(np.abs(line[j:j + len(x)] * weight[:, j]) for j in range(taps))
    if bias is not None:
        y, spread = y + bias, spread + np.abs(bias)
    return (silu(y) if act else y), line[len(x):], spread


def causal_conv_within_bound(got, y, spread):
    """fp32 sums of up to five terms (2^-22 of their sizes; silu's slope is at most 1.1), an exponential and a division of a
    few ulps (2^-20), BF16 (half a step: 2^-8 relative), and silu below -87, which counts as 0."""
    return np.abs(got - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -20 * (np.abs(y) + spread) + 1e-35


def gates(decay, beta, a_log=None, dt_bias=None):
    """(g, beta) of the rule from a call's arrays (rows, heads)."""
    g, b = np.asarray(decay, np.float64), np.asarray(beta, np.float64)
    if a_log is not None:
        g = -np.exp(np.asarray(a_log, np.float64)) * np.logaddexp(g + np.asarray(dt_bias, np.float64), 0.0)
        b = 1.0 / (1.0 + np.exp(-b))
    return np.clip(g, -100.0, 0.0), b


def delta_rule(q, k, v, g, beta, state, scale, normalize=True, wide=False):
    """One sequence: q, k (rows, k_heads, dk), v (rows, heads, dv), g, beta (rows, heads), state (heads, dk, dv). Returns
    (out, state, out_bound, state_bound): the bounds are how far fp32 kernels may be off before out is rounded to BF16.

    State, by columns: a token's arithmetic is fp32 sums of head_k products (2^-19 of the sizes of what is added, also where
    a chunk's products enter the tensor cores as pairs of FP16 parts, 2^-22), through the solve of a chunk (its inverse is a
    contraction's part; 8 times is allowed): eps = 2^-16 of the column's norm and of what the token adds. From then on the
    error is carried by e^g (1 - beta k k^T), which does not stretch while beta |k|^2 is within 0..2.
    Out: the state's error through |q|, the same eps, and the products' own, relative to the magnitudes that are added,
    |q_i| times the state before the chunk and |q_i k_i| |U_j|: operands are fp32 or pairs of FP16 parts (2^-22 each, at most
    two), their decay is good to 2^-21, and a sum of up to 128 and 64 terms takes the tensor cores at most 3 x 12 steps of
    2^-23: 2^-17 in all. (`wide`, for fp32 queries and keys, makes no difference: they are pairs too.)"""
    q, k, v, g, beta = (np.asarray(a, np.float64) for a in (q, k, v, g, beta))
    s = np.asarray(state, np.float64).copy()
    rows, heads, dv = v.shape
    group = heads // k.shape[1]
    if normalize:
        q = q / np.sqrt((q * q).sum(-1, keepdims=True) + UNIT_EPS)
        k = k / np.sqrt((k * k).sum(-1, keepdims=True) + UNIT_EPS)
    q, k = np.repeat(q, group, 1) * scale, np.repeat(k, group, 1)
    eps = 2.0 ** -16
    out, out_bound = np.zeros(v.shape), np.zeros(v.shape)
    off = np.zeros((heads, dv))
    us, upto = [], np.zeros((heads, 0))
    before = np.abs(s)                                            # of the state before the chunk, decayed up to now
    for t in range(rows):
        if t % CHUNK == 0:
            us, ks, upto, before = [], [], np.zeros((heads, 0)), np.abs(s)
        keep = np.exp(g[t])
        s *= keep[:, None, None]
        before = before * keep[:, None, None]
        add = beta[t][:, None] * (v[t] - np.einsum("hk,hkv->hv", k[t], s))
        norm = np.sqrt((s * s).sum(1))
        stretch = np.maximum(1.0, np.abs(1 - beta[t] * (k[t] * k[t]).sum(-1)))[:, None]
        size = np.sqrt((k[t] * k[t]).sum(-1))[:, None]
        off = stretch * keep[:, None] * off + eps * (norm + size * np.abs(beta[t])[:, None] * (np.abs(v[t]) + size * norm))
        s += k[t][:, :, None] * add[:, None, :]
        out[t] = np.einsum("hk,hkv->hv", q[t], s)
        us.append(add)
        ks.append(k[t])
        upto = np.concatenate((upto + g[t][:, None], np.zeros((heads, 1))), 1)
        terms = np.exp(upto) * np.einsum("hk,jhk->hj", np.abs(q[t]), np.abs(np.stack(ks)))
        spread = np.einsum("hk,hkv->hv", np.abs(q[t]), before) + np.einsum("hj,jhv->hv", terms, np.abs(np.stack(us)))
        out_bound[t] = np.sqrt((q[t] * q[t]).sum(-1))[:, None] * (off + eps * norm) + 2.0 ** -17 * spread
    return out, s, out_bound, np.broadcast_to(off[:, None, :], s.shape)


def gated_norm(x, gate, weight, eps):
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    return y if gate is None else y * silu(np.asarray(gate, np.float64))


def gated_norm_within_bound(got, ref):
    """fp32: a sum of up to 256 squares (2^-18 relative covers it with the root, the products and silu's few ulps); BF16: half
    a step (2^-8 relative)."""
    return np.abs(got - ref) <= (2.0 ** -8 + 2.0 ** -17) * np.abs(ref) + 1e-35
