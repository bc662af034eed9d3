"""CPU oracle of the decode step's other operators, plain numpy in fp64: the
4-bit key-value cache's numbers, attention over it, the residual norm and the
sampler's filters. Written from the definitions in include/vbq.h; it shares no
code with the CUDA path."""

from __future__ import annotations

import numpy as np

GROUP = 64
F16_MAX = 65504.0


def kv_quantise(x):
    """x (..., d) -> (codes -7..7, FP16 scales (..., d / 64)) as the cache holds
    them. NaN counts as 0; the quotients and their rounding are exact in fp64
    for fp32 inputs (a 24-bit value over an 11-bit scale)."""
    x = np.where(np.isnan(x), 0.0, np.asarray(x, np.float64))
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    with np.errstate(over="ignore"):
        s = np.minimum(np.abs(g).max(-1) / 7.0, F16_MAX).astype(np.float16)
    sf = s.astype(np.float64)[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(sf > 0, np.clip(np.rint(g / sf), -7, 7), 0.0)
    return q.reshape(x.shape), s


def kv_values(codes, scales):
    g = codes.reshape(*codes.shape[:-1], -1, GROUP) * scales.astype(np.float64)[..., None]
    return g.reshape(codes.shape)


def rotate(x, cos, sin, dtype=np.float32):
    """The pairs (i, i + r / 2) of the first r = 2 cos.shape[-1] dimensions of x
    (rows, heads, d) turned by row, each product and sum rounded to dtype."""
    x, c, s = (np.asarray(a, dtype) for a in (x, cos[:, None, :], sin[:, None, :]))
    h = c.shape[-1]
    out = x.copy()
    a, b = x[..., :h], x[..., h:2 * h]
    out[..., :h] = a * c - b * s
    out[..., h:2 * h] = b * c + a * s
    return out


def attend(q, k, v, pos, scale, window=0, k_scales=None):
    """One sequence: q (rows, heads, d), k and v (tokens, kv_heads, d), pos
    (rows,). Returns (out, spread, reach): spread sums p_j |v_j| and reach is the
    largest scale * sum |q_i| (|k_ji| + 8 s_j) over a row's keys (s_j from
    k_scales, the keys' FP16 scales), for the error bound."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    mag = np.abs(k)
    if k_scales is not None:
        mag = mag + 8.0 * np.repeat(k_scales.astype(np.float64), GROUP, -1)
    rows, heads, d = q.shape
    group = heads // k.shape[1]
    out, spread, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros((rows, heads, 1))
    for r in range(rows):
        lo = max(0, int(pos[r]) - window + 1) if window else 0
        hi = int(pos[r]) + 1
        if hi <= lo:
            continue
        for h in range(heads):
            kk, vv = k[lo:hi, h // group], v[lo:hi, h // group]
            s = kk @ q[r, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h], spread[r, h] = p @ vv, p @ np.abs(vv)
            reach[r, h] = (mag[lo:hi, h // group] @ np.abs(q[r, h])).max() * abs(scale)
    return out, spread, reach


def attend_within_bound(got, out, spread, reach, vmax, tokens):
    """Whether got (BF16 values) is as near as the kernel's roundings allow:
      - probabilities times value scales in FP16: half an ulp, 2^-12, of each
        (twice that allowed), below 2^-14 of the largest an absolute 2^-39 of it
        per key;
      - scores in fp32: their error, at most 2^-19 of sum |q k|, moves a
        probability by twice that (sums of up to 256 products in fp32, and
        codes taken as 0..15 with their middle subtracted);
      - the sum over keys in fp32, of codes 0..15: 2^-19 of 2 vmax;
      - the output's rounding to BF16: 2^-9 of it (twice that allowed)."""
    eps = 2.0 ** -11 + 2.0 * 2.0 ** -19 * reach
    bound = eps * spread + 2.0 ** -8 * np.abs(out) + vmax * (2.0 ** -18 + tokens * 2.0 ** -38)
    return np.abs(got - out) <= bound


def residual_norm(x, residual, weight, eps, round_residual):
    """(out, r') with r' = round_residual(residual + x), fp64 otherwise."""
    r = np.asarray(x, np.float64) if residual is None else \
        round_residual((np.asarray(residual, np.float64) + np.asarray(x, np.float64)).astype(np.float32)).astype(np.float64)
    return r / np.sqrt((r * r).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64), r


def sample_filters(logits, temperature, top_k, top_p, min_p):
    """One row: (weights e_i of the kept tokens, 0 elsewhere; kept mask; edge),
    edge the smallest relative distance of a top-p or min-p decision to its
    threshold (the fp32 kernel may decide the other way when it is tiny)."""
    l = np.asarray(logits, np.float64).copy()
    l[np.isnan(l)] = -np.inf
    top = l.max()
    if top == -np.inf:
        return np.zeros_like(l), np.zeros(l.shape, bool), np.inf
    order = np.argsort(-l, kind="stable")
    if not temperature > 0:
        e = np.zeros_like(l)
        e[order[0]] = 1.0
        return e, e > 0, np.inf
    with np.errstate(invalid="ignore"):
        e = np.where(l == top, 1.0, np.exp(np.where(l == -np.inf, -np.inf, l - top) / np.float64(temperature)))
    edge = np.inf
    if top_k > 0:
        order = order[:top_k]
    if not top_p >= 1:
        mass = e[order].cumsum()
        want = max(float(top_p), 0.0) * mass[-1]
        n = int((mass < want).sum()) + 1
        edge = min(edge, np.abs(mass - want).min() / mass[-1])
        order = order[:n]
    keep = e[order] >= min(float(min_p), 1.0)
    if min_p > 0:
        edge = min(edge, np.abs(e[order][e[order] < 1] - min_p).min(initial=np.inf) / min_p)
    order = order[keep & (l[order] > -np.inf)]
    mask = np.zeros(l.shape, bool)
    mask[order] = True
    return np.where(mask, e, 0.0), mask, edge


def sample_weights(logits, temperature):
    """One row, on the whole weights that the sampler's definition gives: (order, low, high), the tokens above -inf from
    the largest logit down, equal ones by index, and the least and the largest whole number of 2^-32 that each may weigh.
    e = exp((l - m) / T) is of fp32: l - m is rounded once, 2^-24 of the exponent; the rest of the exponent's arithmetic
    (2^-24) and a base-2 exponential good to 2 ulps (2^-22) come on top. Twice that is allowed: 2^-23 (|exponent| + 8)."""
    l = np.asarray(logits, np.float64).copy()
    l[np.isnan(l)] = -np.inf
    order = np.argsort(-l, kind="stable")
    order = order[l[order] > -np.inf]
    x = (l[order] - l[order[0]]) / np.float64(temperature)
    e, slack = np.exp(x), np.minimum(2.0 ** -23 * (np.abs(x) + 8.0), 1.0)
    return order, np.rint(e * (1 - slack) * 2.0 ** 32), np.rint(np.minimum(e * (1 + slack), 1.0) * 2.0 ** 32)


def sample_kept(low, high, top_k, top_p, min_p):
    """How many tokens of sample_weights' order the filters may leave, at least and at most (each filter leaves a run from
    the first one on)."""
    n = len(low)
    k = min(top_k, n) if top_k > 0 else n
    a = b = k
    if not top_p >= 1:
        p = max(float(top_p), 0.0) if top_p == top_p else 0.0
        lows, highs = low[:k].cumsum(), high[:k].cumsum()
        a = int((highs < p * lows[-1]).sum()) + 1
        b = min(int((lows < p * highs[-1]).sum()) + 1, k)
    m = min(float(min_p), 1.0) * 2.0 ** 32
    if m > 0:
        a = min(a, max(int((low[:k] >= m + 1).sum()), 1))
        b = min(b, max(int((high[:k] + 1 >= m).sum()), 1))
    return a, b


def sample_drawn_ok(order, low, high, temperature, logits, u, token, prob, kept):
    """Whether token and prob are the draw among the first `kept` tokens of order: the kept weights before the token, at
    their least, are at most u times all of them at their most, those up to it, at their most, more than u times all at
    their least; prob is its weight's share, one rounding of each of its terms and of the quotient (2^-22) aside."""
    at = np.flatnonzero(order[:kept] == token)
    if at.size != 1:
        return False
    at = at[0]
    lo, hi = low[:kept], high[:kept]
    before = order[:kept] < token
    if not (lo[before].sum() <= u * hi.sum() and hi[before].sum() + hi[at] > u * lo.sum()):
        return False
    l = np.asarray(logits, np.float64)
    x = (l[token] - l[order[0]]) / np.float64(temperature)
    e, slack = np.exp(x) * 2.0 ** 32, 2.0 ** -23 * (abs(x) + 8.0)
    return e * (1 - slack) / hi.sum() * (1 - 2.0 ** -22) <= prob <= e * (1 + slack) / lo.sum() * (1 + 2.0 ** -22)
