"""The operators of a linear-attention layer (vbq_causal_conv, vbq_delta_rule,
vbq_gated_norm) against the fp64 oracle, through the C ABI."""

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import delta_oracle as o

pytestmark = pytest.mark.gpu

DEV, I32, BF16, F32 = "cuda", torch.int32, torch.bfloat16, torch.float32
JUNK = 7.0


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


def np64(t):
    return t.double().cpu().numpy()


def dev(a, dtype=F32):
    return torch.from_numpy(np.asarray(a)).to(DEV).to(dtype)


def starts_of(lens, first=0):
    return np.concatenate(([0], np.cumsum(lens))).astype(np.int32) + first


def sequences(lens, slots, fresh=None, first=0, behind=0, rows=None):
    """Packed after `first` rows of no sequence and before `behind` more."""
    s = starts_of(lens, first)
    return vbq.Sequences(len(lens), max(lens) if rows is None else rows, starts=dev(s, I32), tokens=int(s[-1]) + behind, slots=dev(np.array(slots), I32),
                         fresh=None if fresh is None else dev(np.array(fresh), I32))


# ---------------------------------------------------------------------------
# convolution
# ---------------------------------------------------------------------------

def run_conv(lens, channels, taps, dtype, bias=True, act=True, idle=(), fresh=(), pad=0, uniform=False, seed=0):
    rng = np.random.default_rng(seed + channels + taps)
    first, behind = (0, 0) if uniform else (3, 2)
    tokens = sum(lens) + first + behind
    wide = dev(rng.standard_normal((tokens, channels + pad)).astype(np.float32), dtype)
    x = wide[:, pad // 2:pad // 2 + channels]
    w, b = (rng.standard_normal(s).astype(np.float32) for s in ((channels, taps), channels))
    n_slots = len(lens) + 2
    slots = rng.permutation(n_slots)[:len(lens)].astype(np.int32)
    for i in idle:
        slots[i] = -1 - i
    state = dev(rng.standard_normal((n_slots, taps - 1, channels)).astype(np.float32))
    before = np64(state)
    flags = [int(i in fresh) for i in range(len(lens))]
    if uniform:
        seq = vbq.Sequences(len(lens), lens[0], slots=dev(slots, I32), fresh=dev(flags, I32))
    else:
        seq = sequences(lens, slots, flags, first, behind)
    out = torch.full((tokens, channels), JUNK, dtype=BF16, device=DEV)
    vbq.vbq_causal_conv(seq, x, dev(w), state, bias=dev(b) if bias else None, silu=act, out=out)
    got, after, xs = np64(out), np64(state), np64(x)
    want = before.copy()
    at = first
    assert (got[:first] == JUNK).all() and (got[tokens - behind:] == JUNK).all()
    for i, n in enumerate(lens):
        if slots[i] < 0:
            assert not got[at:at + n].any()
        elif n:
            past = np.zeros_like(before[0]) if flags[i] else before[slots[i]]
            y, last, spread = o.causal_conv(xs[at:at + n], w, past, b if bias else None, act)
            assert o.causal_conv_within_bound(got[at:at + n], y, spread).all(), f"sequence {i}"
            want[slots[i]] = last
        at += n
    assert np.array_equal(after, want)                            # inputs are carried as they are, other slots untouched
    return out


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("taps", [2, 3, 4])
@pytest.mark.parametrize("channels,pad", [(8, 0), (1000, 32), (2056, 0)], ids=str)
def test_conv_matches_oracle(channels, pad, taps, dtype):
    run_conv([1, 0, 2, 3, 4, 31, 32, 33, 64, 65, 0, 1, 100], channels, taps, dtype, idle=(4, 8), fresh=(2, 6, 11), pad=pad)


def test_conv_of_uniform_rows_without_bias_or_silu():
    for rows in (1, 2, 40):
        run_conv([rows] * 5, 256, 4, F32, bias=False, act=False, fresh=(1,), uniform=True)


def test_conv_of_many_sequences():
    """Lookup of a tile's sequence over more than 32 and more than 1024 of them, empty ones among them."""
    rng = np.random.default_rng(5)
    run_conv([int(n) for n in rng.integers(0, 4, 40)], 64, 4, BF16)
    run_conv([int(n) for n in rng.integers(0, 3, 1500)], 16, 4, F32)
    run_conv([0] * 1100 + [70] + [0] * 200 + [1], 16, 3, F32)


def test_conv_cut_anywhere_is_the_same():
    rng = np.random.default_rng(1)
    x, w = dev(rng.standard_normal((90, 64)).astype(np.float32)), dev(rng.standard_normal((64, 4)).astype(np.float32))
    state = torch.zeros(1, 3, 64, device=DEV)
    whole = vbq.vbq_causal_conv(vbq.Sequences(1, 90), x, w, state)
    for cuts in ([1] * 90, [2, 1, 87], [32, 33, 25], [5, 64, 21]):
        part, at, outs = torch.zeros(1, 3, 64, device=DEV), 0, []
        for n in cuts:
            outs.append(vbq.vbq_causal_conv(vbq.Sequences(1, n), x[at:at + n], w, part))
            at += n
        assert torch.equal(torch.cat(outs), whole) and torch.equal(part, state)


def test_conv_extremes():
    """Infinities and NaN stay in their channel and within the window; what a fresh sequence's slot held does not matter."""
    x = torch.randn(40, 64, device=DEV)
    w = torch.randn(64, 4, device=DEV)
    state = torch.full((1, 3, 64), float("nan"), device=DEV)
    fresh = torch.ones(1, dtype=I32, device=DEV)
    want = vbq.vbq_causal_conv(vbq.Sequences(1, 40, fresh=fresh), x, w, state.clone())
    assert torch.isfinite(want).all()
    x[10, 7], x[20, 9], x[30, 1] = float("nan"), float("inf"), -1e38
    got = vbq.vbq_causal_conv(vbq.Sequences(1, 40, fresh=fresh), x, w, state)
    bad = torch.zeros(40, 64, dtype=torch.bool, device=DEV)
    bad[10:14, 7], bad[20:24, 9], bad[30:34, 1] = True, True, True
    assert torch.equal(got[~bad], want[~bad]) and torch.isnan(got[10:14, 7]).all() and torch.isfinite(state).all()


# ---------------------------------------------------------------------------
# delta rule
# ---------------------------------------------------------------------------

def inputs(rng, tokens, hk, h, dk, dv, dtype, raw, gate_dtype=F32, pad=16, sizes=1.0):
    """q, k and v as slices of one array, gates as slices of another."""
    wide = dev((rng.standard_normal((tokens, 2 * hk * dk + h * dv + pad)) * sizes).astype(np.float32), dtype)
    q, k, v = (wide[:, a:a + n * d].unflatten(1, (n, d)) for a, n, d in ((0, hk, dk), (hk * dk, hk, dk), (2 * hk * dk, h, dv)))
    gates = rng.standard_normal((tokens, 2 * h + 3)).astype(np.float32)
    if raw:
        a_log, dt = np.log(rng.uniform(0.5, 16, h)).astype(np.float32), rng.uniform(-6, 0, h).astype(np.float32)
    else:
        a_log = dt = None
        gates[:, :h] = -np.exp(2 * gates[:, :h] - 3)
        gates[:, h + 1:2 * h + 1] = 1 / (1 + np.exp(-gates[:, h + 1:2 * h + 1]))
    gates = dev(gates, gate_dtype)
    return q, k, v, gates[:, :h], gates[:, h + 1:2 * h + 1], a_log, dt


def check_delta(got, after, before, lens, slots, flags, first, q, k, v, a, b, a_log, dt, scale, normalize=True, lasting=()):
    got, after, before = np64(got), np64(after), np64(before)
    g, beta = o.gates(np64(a), np64(b), a_log, dt)
    wide = v.dtype == F32
    q, k, v = np64(q), np64(k), np64(v)
    want, bound, at = before.copy(), np.zeros_like(before), first
    for i, n in enumerate(lens):
        s = slice(at, at + n)
        if slots[i] < 0:
            assert not got[s].any()
        elif n:
            start = np.zeros_like(before[0]) if flags[i] else before[slots[i]]
            out, end, ob, sb = o.delta_rule(q[s], k[s], v[s], g[s], beta[s], start, scale, normalize, wide)
            off = np.abs(got[s] - out) - (ob + 2.0 ** -8 * (np.abs(out) + ob))
            assert (off <= 0).all(), f"out of sequence {i} ({n} rows): {off.max():.3g} outside"
            want[slots[i]], bound[slots[i]] = end, sb
        at += n
    off = np.abs(after - want) - bound
    assert (off <= 0).all(), f"state: {off.max():.3g} outside"
    # Of fp32 throughout; a part held in 16 bits would show. Where the rule contracts, that is: with beta |k|^2 = 2 an error
    # lasts (the map is a reflection), so n tokens of 2^-24 times some 19 additions each may add up to n 2^-20, and only the
    # bound above holds for such heads (`lasting`).
    heads = [i for i in range(after.shape[1]) if i not in lasting]
    assert np.linalg.norm((after - want)[:, heads]) <= 2.0 ** -17 * np.linalg.norm(want[:, heads])


def run_delta(lens, hk, h, dk, dv, dtype=BF16, raw=True, gate_dtype=F32, idle=(), fresh=(), normalize=True, uniform=False, seed=0, rows=None, sizes=1.0):
    rng = np.random.default_rng(seed + 7 * h + dk + dv)
    first, behind = (0, 0) if uniform else (2, 3)
    tokens = sum(lens) + first + behind
    q, k, v, a, b, a_log, dt = inputs(rng, tokens, hk, h, dk, dv, dtype, raw, gate_dtype, sizes=sizes)
    if not normalize:
        q, k = (q.float() * dk ** -0.5).to(dtype), (k.float() * dk ** -0.5).to(dtype)
    n_slots = len(lens) + 2
    slots = rng.permutation(n_slots)[:len(lens)].astype(np.int32)
    for i in idle:
        slots[i] = -1
    flags = [int(i in fresh) for i in range(len(lens))]
    state = dev(rng.standard_normal((n_slots, h, dk, dv)).astype(np.float32) * 0.5)
    before = state.clone()
    if uniform:
        seq = vbq.Sequences(len(lens), lens[0], slots=dev(slots, I32), fresh=dev(flags, I32))
    else:
        seq = sequences(lens, slots, flags, first, behind, rows)
    out = torch.full((tokens, h, dv), JUNK, dtype=BF16, device=DEV)
    par = dict(a_log=None if a_log is None else dev(a_log), dt_bias=None if dt is None else dev(dt), normalize=normalize)
    vbq.vbq_delta_rule(seq, state, q, k, v, a, b, out=out, **par)
    assert (out[:first] == JUNK).all() and (out[tokens - behind:] == JUNK).all()
    check_delta(out, state, before, lens, slots, flags, first, q, k, v, a, b, a_log, dt, dk ** -0.5, normalize)
    # the same call again gives the same bits
    again, two = before.clone(), torch.full_like(out, JUNK)
    vbq.vbq_delta_rule(seq, again, q, k, v, a, b, out=two, **par)
    assert torch.equal(again, state) and torch.equal(two, out)


LENS = [1, 0, 2, 63, 64, 65, 17, 129, 5, 0, 200, 1]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("hk,h,dk,dv", [(1, 1, 64, 64), (2, 2, 128, 128), (1, 3, 128, 64), (2, 4, 64, 256), (1, 2, 128, 256), (3, 3, 64, 128)], ids=str)
def test_delta_matches_oracle(hk, h, dk, dv, dtype):
    run_delta(LENS, hk, h, dk, dv, dtype, idle=(3, 8), fresh=(2, 7))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_delta_with_gates_of_the_caller_s(dtype):
    run_delta(LENS, 2, 4, 128, 128, dtype, raw=False, fresh=(0,))
    run_delta([70, 3], 2, 2, 64, 64, dtype, raw=False, gate_dtype=BF16, normalize=False)


def test_delta_of_uniform_rows():
    for rows in (1, 3, 16, 80):
        run_delta([rows] * 5, 2, 4, 128, 128, fresh=(1,), uniform=True)


def test_delta_of_a_longest_that_is_not():
    """`rows` only says what to expect: longer sequences are computed all the same."""
    run_delta([3, 150, 1], 1, 2, 128, 64, rows=1)
    run_delta([3, 2, 1], 1, 2, 128, 64, rows=5000)


def test_delta_of_a_long_sequence():
    run_delta([1500], 1, 2, 128, 128, raw=True, seed=3)
    run_delta([1111], 1, 1, 64, 64, F32, raw=False, seed=3)


@pytest.mark.parametrize("sizes", [1e-12, 1e12], ids=str)
def test_delta_of_small_and_large_values(sizes):
    """Unit length takes the sizes of q and k away (but for its epsilon); v's pass through."""
    run_delta([1, 70, 20], 1, 2, 128, 64, sizes=sizes)
    run_delta([1, 70, 20], 1, 2, 64, 64, F32, sizes=sizes)


@pytest.mark.parametrize("rows", [9, 100])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_delta_at_the_edges_of_its_gates(rows, dtype):
    """No decay and all of it (alone, and in the middle of a chunk), betas 0, 1 and 2, one key for every token, keys and
    queries of zeros, an empty state."""
    rng = np.random.default_rng(rows)
    h, d = 8, 64
    q, k, v, a, b, _, _ = inputs(rng, rows, h, h, d, d, dtype, False)
    q, k, v, a, b = (t.clone() for t in (q, k, v, a, b))
    a[:, 0], b[:, 0] = 0.0, 1.0                                   # keeps everything, overwrites whole keys
    a[:, 1], b[:, 1] = -100.0, 1.0                                # keeps nothing
    a[rows // 2, 2], a[rows // 2 + 2, 2] = -1000.0, float("-inf")  # forgets twice within a chunk
    b[:, 3] = 0.0                                                 # learns nothing
    a[:, 4], b[:, 4], k[:, 4] = 0.0, 1.0, k[0, 4]                 # one key
    a[:, 5], b[:, 5], k[:, 5] = 0.0, 2.0, k[0, 5] * torch.where(torch.arange(rows, device=DEV) % 2 == 0, 1.0, -1.0)[:, None].to(dtype)
    k[:, 6] = 0
    q[:, 6] = 0
    a[:, 7] = 3.0                                                 # counts as 0
    state = torch.randn(1, h, d, d, device=DEV)
    state[0, 0] = 0
    before = state.clone()
    out = vbq.vbq_delta_rule(vbq.Sequences(1, rows), state, q, k, v, a, b)
    check_delta(out, state, before, [rows], [0], [0], 0, q, k, v, a, b, None, None, d ** -0.5, lasting=(5,))
    assert not out[:, 6].any()


def test_delta_gates_of_large_inputs():
    """softplus and sigmoid far out on both sides."""
    rng = np.random.default_rng(2)
    q, k, v, a, b, _, _ = inputs(rng, 90, 2, 2, 64, 64, BF16, True)
    a, b = a.clone(), b.clone()
    a[::5, 0], a[1::5, 0], b[::4, 1], b[1::4, 1] = 300.0, -300.0, 200.0, -200.0
    a_log, dt = np.array([-2.0, 1.0], np.float32), np.array([0.5, -0.5], np.float32)
    state = torch.randn(1, 2, 64, 64, device=DEV)
    before = state.clone()
    out = vbq.vbq_delta_rule(vbq.Sequences(1, 90), state, q, k, v, a, b, a_log=dev(a_log), dt_bias=dev(dt))
    check_delta(out, state, before, [90], [0], [0], 0, q, k, v, a, b, a_log, dt, 0.125)


@pytest.mark.parametrize("rows", [4, 130])
def test_delta_nan_stays_in_its_head_and_column(rows):
    """A NaN or an infinity of a value reaches its column alone, of a gate its head; a fresh state's slot may hold anything."""
    rng = np.random.default_rng(rows)
    q, k, v, a, b, _, _ = inputs(rng, 2 * rows, 4, 4, 128, 64, BF16, False)
    q, k, v, a, b = (t.clone() for t in (q, k, v, a, b))
    fresh = torch.ones(2, dtype=I32, device=DEV)
    nan = lambda: torch.full((2, 4, 128, 64), float("nan"), device=DEV)  # noqa: E731
    seq, ws = vbq.Sequences(2, rows, fresh=fresh), nan()
    want = vbq.vbq_delta_rule(seq, ws, q, k, v, a, b)
    assert torch.isfinite(want).all() and torch.isfinite(ws).all()
    v[rows + 1, 0, 5] = float("nan")
    v[2, 1, 9] = float("inf")
    a[3, 2] = float("nan")
    gs = nan()
    got = vbq.vbq_delta_rule(seq, gs, q, k, v, a, b)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[rows + 1:, 0, 5], bad[:rows, 1, 9], bad[:rows, 2] = True, True, True
    first = bad.clone()                                           # rows before the value: causal, but a chunk may share their column
    assert torch.equal(got[~bad], want[~bad]) and torch.isnan(got[rows + 1:, 0, 5]).all() and torch.isnan(got[3:rows, 2]).all()
    keep = torch.ones_like(gs, dtype=torch.bool)
    keep[1, 0, :, 5], keep[0, 1, :, 9], keep[0, 2] = False, False, False
    assert torch.equal(gs[keep], ws[keep]) and torch.isnan(gs[1, 0, :, 5]).all()
    del first


@pytest.mark.parametrize("rows,at", [(1, 0), (12, 5), (20, 5), (130, 0), (130, 5), (130, 22), (130, 77), (130, 127)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_delta_nan_reaches_no_earlier_token(rows, at, dtype):
    """One token's key, query, decay or factor is NaN or infinite, a head each: what comes before is as without it, what comes
    after is NaN (of a query: that token alone)."""
    rng = np.random.default_rng(at)
    h, dk, dv = 6, 128, 64
    q, k, v, a, b, _, _ = inputs(rng, rows, h, h, dk, dv, dtype, False)
    q, k, v, a, b = (t.clone() for t in (q, k, v, a, b))
    clean = [np64(t) for t in (q, k, v, a, b)]
    k[at, 0, 3], k[at, 1, 100], q[at, 2, 64], a[at, 3], b[at, 4], k[at, 5, 7] = (float(x) for x in ("nan", "inf", "nan", "nan", "inf", "-inf"))
    state = torch.randn(1, h, dk, dv, device=DEV)
    before = np64(state)[0]
    got = np64(vbq.vbq_delta_rule(vbq.Sequences(1, rows), state, q, k, v, a, b))
    after = np64(state)[0]
    g, beta = o.gates(clean[3], clean[4], None, None)
    want, end, bound, sb = o.delta_rule(clean[0], clean[1], clean[2], g, beta, before, dk ** -0.5, True, dtype == F32)
    off = np.abs(got - want) - (bound + 2.0 ** -8 * (np.abs(want) + bound))
    assert (off[:at] <= 0).all(), f"heads {np.unique(np.argwhere(~(off[:at] <= 0))[:, 1])}"
    assert (off[at + 1:, 2] <= 0).all() and (np.abs(after[2] - end[2]) <= sb[2]).all() and np.isnan(got[at, 2]).all()
    lost = [0, 1, 3, 4, 5]
    assert not np.isfinite(got[at:, lost]).any() and not np.isfinite(after[lost]).any()


# Sequences and heads so many that 64 columns of a state go to a block instead of 32 (where a head's 32 would take a second
# round of blocks and its 64 do not), idle, fresh and empty ones among them.
@pytest.mark.parametrize("lens,hk,h,dk,dv", [([130, 129, 1, 0, 140, 130, 128], 8, 16, 128, 128), ([65, 64, 90, 63, 80], 16, 16, 64, 128),
                                             ([200, 170], 16, 32, 128, 128), ([100] * 11, 8, 8, 64, 64)], ids=str)
def test_delta_of_wide_blocks(lens, hk, h, dk, dv):
    run_delta(lens, hk, h, dk, dv, idle=(1,), fresh=(0, len(lens) - 1))
    run_delta(lens, hk, h, dk, dv, raw=False, gate_dtype=BF16, fresh=(0,))


def test_delta_of_short_and_long_sequences_in_turn():
    """Calls one after the other whose short sequences are the next call's long ones: the kernels of a call run side by side,
    those of two calls must not. Bit for bit what calls with a wait in between give, in a graph too."""
    rng = np.random.default_rng(11)
    h, d, steps = 8, 128, 12
    calls = []
    for i in range(steps):
        lens = [int(n) for n in np.where(np.arange(20) % 2 == i % 2, rng.integers(1, 25, 20), rng.integers(25, 150, 20))]
        q, k, v, a, b, a_log, dt = inputs(rng, sum(lens), h, h, d, d, BF16, True)
        par = dict(a_log=dev(a_log), dt_bias=dev(dt), out=torch.empty(sum(lens), h, d, dtype=BF16, device=DEV))
        calls.append((sequences(lens, rng.permutation(20).astype(np.int32) if i % 3 == 0 else np.arange(20)), (q, k, v, a, b), par))
    start = torch.randn(20, h, d, d, device=DEV)

    def run(state, wait):
        for seq, x, par in calls:
            vbq.vbq_delta_rule(seq, state, *x, **par)
            if wait:
                torch.cuda.synchronize()
        return [par["out"].clone() for _, _, par in calls]

    want_state = start.clone()
    want = run(want_state, True)
    state = start.clone()
    got = run(state, False)
    assert torch.equal(state, want_state) and all(map(torch.equal, got, want))
    graph, state = torch.cuda.CUDAGraph(), start.clone()
    with torch.cuda.graph(graph):
        run(state, False)
    for _ in range(3):
        state.copy_(start)
        graph.replay()
        assert torch.equal(state, want_state) and all(torch.equal(par["out"], w) for (_, _, par), w in zip(calls, want))


def test_delta_cut_anywhere_is_the_same_to_rounding():
    rng = np.random.default_rng(8)
    n, hk, h, d = 333, 1, 2, 128
    q, k, v, a, b, a_log, dt = inputs(rng, n, hk, h, d, d, BF16, True)
    g, beta = o.gates(np64(a), np64(b), a_log, dt)
    ref, end, ob, sb = o.delta_rule(np64(q), np64(k), np64(v), g, beta, np.zeros((h, d, d)), d ** -0.5)
    par = dict(a_log=dev(a_log), dt_bias=dev(dt))
    for cuts in ([333], [1] * 20 + [313], [64, 64, 205], [100, 1, 232], [3, 16, 16, 16, 16, 16, 250]):
        state, at, outs = torch.zeros(1, h, d, d, device=DEV), 0, []
        for m in cuts:
            s = slice(at, at + m)
            outs.append(vbq.vbq_delta_rule(vbq.Sequences(1, m), state, q[s], k[s], v[s], a[s], b[s], **par))
            at += m
        assert (np.abs(np64(state)[0] - end) <= sb).all()
        # the bound on what a chunk rounds goes by chunks from the first row on; twice it covers other cuts
        assert (np.abs(np64(torch.cat(outs)) - ref) <= 2 * ob + 2.0 ** -8 * (np.abs(ref) + ob)).all()


def test_slots_outside_the_pool_are_reported():
    x = torch.randn(6, 64, device=DEV)
    w = torch.randn(64, 4, device=DEV)
    slots = torch.tensor([0, 9, 1], dtype=I32, device=DEV)
    conv_state = torch.randn(2, 3, 64, device=DEV)
    assert vbq.vbq_device_status() is None
    out = vbq.vbq_causal_conv(vbq.Sequences(3, 2, slots=slots), x, w, conv_state)
    assert out[:2].any() and not out[2:4].any() and out[4:].any()
    with pytest.raises(vbq.VbqError, match="pool"):
        vbq.vbq_device_status()
    for rows in (2, 100):
        q = torch.randn(3 * rows, 1, 64, device=DEV).to(BF16)
        gate = torch.zeros(3 * rows, 1, device=DEV)
        state = torch.randn(2, 1, 64, 64, device=DEV)
        out = vbq.vbq_delta_rule(vbq.Sequences(3, rows, slots=slots), state, q, q, q, gate, gate + 0.5)
        assert out[:rows].any() and not out[rows:2 * rows].any() and out[2 * rows:].any()
        with pytest.raises(vbq.VbqError, match="pool"):
            vbq.vbq_device_status()
        assert vbq.vbq_device_status() is None
    # without slots the sequence's number is its slot
    vbq.vbq_causal_conv(vbq.Sequences(3, 2), x, w, conv_state)
    with pytest.raises(vbq.VbqError, match="pool"):
        vbq.vbq_device_status()


def test_starts_outside_the_rows_stay_within_them():
    """Whatever starts holds, no row outside 0..tokens is touched."""
    rows, h, d, c = 40, 2, 64, 64
    big = torch.full((rows + 200, h, d), JUNK, dtype=BF16, device=DEV)
    conv_big = torch.full((rows + 200, c), JUNK, dtype=BF16, device=DEV)
    q = torch.randn(rows, h, d, device=DEV).to(BF16)
    gate = torch.zeros(rows, h, device=DEV)
    x, w = torch.randn(rows, c, device=DEV), torch.randn(c, 4, device=DEV)
    for starts in ([-50, 10, 500], [30, 20, 35], [1000, 2000, 3000], [-9, -8, -7], [39, 41, 43]):
        seq = vbq.Sequences(2, 500, starts=torch.tensor(starts, dtype=I32, device=DEV), tokens=rows)
        big.fill_(JUNK)
        conv_big.fill_(JUNK)
        vbq.vbq_delta_rule(seq, torch.zeros(2, h, d, d, device=DEV), q, q, q, gate, gate + 0.5, out=big[100:100 + rows])
        vbq.vbq_causal_conv(seq, x, w, torch.zeros(2, 3, c, device=DEV), out=conv_big[100:100 + rows])
        for t in (big, conv_big):
            assert (t[:100] == JUNK).all() and (t[100 + rows:] == JUNK).all()


def test_states_beyond_32_bit_offsets():
    """A pool of more than 2^31 floats, a call's rows beyond 2^31 elements."""
    h, d = 32, 128
    n_slots = 4200                                                # x 32 x 128 x 128 floats: 8.8 GB
    state = torch.empty(n_slots, h, d, d, device=DEV)
    rng = np.random.default_rng(4)
    for lens in ([1, 2], [70, 3]):
        tokens = sum(lens)
        q, k, v, a, b, a_log, dt = inputs(rng, tokens, 16, h, d, d, BF16, True)
        slots = [n_slots - 1, 4110]
        state[slots] = torch.randn(2, h, d, d, device=DEV)
        before = state[slots].clone()
        out = vbq.vbq_delta_rule(sequences(lens, slots), state, q, k, v, a, b, a_log=dev(a_log), dt_bias=dev(dt))
        heads = [0, 31]
        pick = lambda t: t[:, heads]  # noqa: E731
        check_delta(pick(out), state[slots][:, heads], before[:, heads], lens, [0, 1], [0, 0], 0, q[:, [0, 15]], k[:, [0, 15]], pick(v), pick(a), pick(b),
                    a_log[heads], dt[heads], d ** -0.5)
    del state
    rows, c = 270000, 8192
    x = torch.randn(512, c, device=DEV).to(BF16).repeat(rows // 512 + 1, 1)[:rows].contiguous()
    w = torch.randn(c, 4, device=DEV)
    out = vbq.vbq_causal_conv(vbq.Sequences(1, rows), x, w, torch.zeros(1, 3, c, device=DEV))
    y, _, spread = o.causal_conv(np64(x[-100:]), np64(w), np64(x[-103:-100]))
    assert o.causal_conv_within_bound(np64(out[-100:]), y, spread).all()
    gate = torch.randn(1, c, device=DEV).to(BF16).expand(rows, -1).contiguous()
    n = vbq.vbq_gated_norm(x.unflatten(1, (64, 128)), gate.unflatten(1, (64, 128)), torch.ones(128, device=DEV), 1e-6)
    ref = o.gated_norm(np64(x[-3:]).reshape(3, 64, 128), np64(gate[-3:]).reshape(3, 64, 128), np.ones(128), 1e-6)
    assert o.gated_norm_within_bound(np64(n[-3:]), ref).all()


# ---------------------------------------------------------------------------
# gated norm
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("rows,heads,width", [(1, 1, 8), (3, 5, 64), (7, 32, 128), (2, 3, 256), (300, 12, 72), (5, 2, 200)], ids=str)
@pytest.mark.parametrize("x_type", [F32, BF16], ids=["xf32", "xbf16"])
@pytest.mark.parametrize("gate", [F32, BF16, None], ids=["zf32", "zbf16", "none"])
def test_gated_norm_matches_oracle(rows, heads, width, x_type, gate):
    rng = np.random.default_rng(rows + width)
    wide = lambda t: dev((rng.standard_normal((rows, heads * width + 24)) * 3).astype(np.float32), t)[:, 8:8 + heads * width].unflatten(1, (heads, width))  # noqa: E731
    x, z = wide(x_type), None if gate is None else wide(gate)
    w = rng.standard_normal(width).astype(np.float32)
    out = vbq.vbq_gated_norm(x, z, dev(w), 1e-6)
    assert o.gated_norm_within_bound(np64(out), o.gated_norm(np64(x), None if z is None else np64(z), w, 1e-6)).all()


def test_gated_norm_in_place_empty_and_extremes():
    w = torch.ones(64, device=DEV)
    assert vbq.vbq_gated_norm(torch.zeros(0, 3, 64, device=DEV), None, w, 1e-6).shape == (0, 3, 64)
    assert not vbq.vbq_gated_norm(torch.zeros(2, 3, 64, device=DEV), None, w, 1e-6).any()
    x, z = torch.randn(50, 3, 64, device=DEV).to(BF16), torch.randn(50, 3, 64, device=DEV)
    want = vbq.vbq_gated_norm(x, z, w, 1e-6)
    x[4, 1, 9], z[7, 2, 5], z[8, 0, 3], z[9, 1, 1] = float("nan"), -500.0, 500.0, float("-inf")
    same = x.clone()
    got = vbq.vbq_gated_norm(same, z, w, 1e-6, out=same)
    assert got is same and torch.isnan(got[4, 1]).all() and got[7, 2, 5] == 0 and torch.isfinite(got[8, 0, 3])
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[4, 1], bad[7, 2, 5], bad[8, 0, 3], bad[9, 1, 1] = True, True, True, True
    assert torch.equal(got[~bad], want[~bad])


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

class Layer:
    """The three operators as a layer uses them: from one product's fp32 output (q, k, v channels, gate, decay, beta) a token
    to the next product's BF16 input."""

    def __init__(self, rng, hk, h, d, slots):
        self.hk, self.h, self.d = hk, h, d
        self.channels = (2 * hk + h) * d
        self.w = dev(rng.standard_normal((self.channels, 4)).astype(np.float32) * 0.5)
        self.a_log = dev(np.log(rng.uniform(1, 16, h)).astype(np.float32))
        self.dt = dev(rng.uniform(-6, -2, h).astype(np.float32))
        self.norm = dev(rng.uniform(0.5, 1.5, d).astype(np.float32))
        self.conv_state = torch.zeros(slots, 3, self.channels, device=DEV)
        self.state = torch.zeros(slots, h, d, d, device=DEV)
        self.width = self.channels + h * d + 2 * h

    def __call__(self, seq, y, stream=None):
        hk, h, d, c = self.hk, self.h, self.d, self.channels
        x = vbq.vbq_causal_conv(seq, y[:, :c], self.w, self.conv_state, stream=stream)
        q, k, v = (x[:, a:a + n * d].unflatten(1, (n, d)) for a, n in ((0, hk), (hk * d, hk), (2 * hk * d, h)))
        z, a, b = y[:, c:c + h * d].unflatten(1, (h, d)), y[:, c + h * d:c + h * d + h], y[:, c + h * d + h:]
        out = vbq.vbq_delta_rule(seq, self.state, q, k, v, a, b, a_log=self.a_log, dt_bias=self.dt, stream=stream)
        return vbq.vbq_gated_norm(out, z, self.norm, 1e-6, stream=stream)

    def reference(self, y, lens):
        """Token by token in fp64 from empty states, rounded to BF16 where the layer does."""
        hk, h, d, c = self.hk, self.h, self.d, self.channels
        y, outs, at = np64(y), [], 0
        bf16 = lambda a: torch.from_numpy(a).to(BF16).double().numpy()  # noqa: E731
        for n in lens:
            r = y[at:at + n]
            x = bf16(o.causal_conv(r[:, :c], np64(self.w), np.zeros((3, c)))[0])
            g, beta = o.gates(r[:, c + h * d:c + h * d + h], r[:, c + h * d + h:], np64(self.a_log), np64(self.dt))
            q, k, v = (x[:, i:i + m * d].reshape(n, m, d) for i, m in ((0, hk), (hk * d, hk), (2 * hk * d, h)))
            out = o.delta_rule(q, k, v, g, beta, np.zeros((h, d, d)), d ** -0.5)[0]
            outs.append(o.gated_norm(bf16(out), r[:, c:c + h * d].reshape(n, h, d), np64(self.norm), 1e-6))
            at += n
        return np.concatenate(outs)


def test_layer_prompt_then_tokens():
    """Prompts of different lengths, then single tokens of all sequences in one captured graph, against fp64 over the whole.
    Each of the three roundings to BF16 (2^-9 relative and independent, so 2^-8 of the norm together) is in the reference
    too, but now and then falls the other way: 1% of the norm is allowed."""
    rng = np.random.default_rng(11)
    layer, lens, steps = Layer(rng, 2, 4, 64, 6), [70, 1, 130, 9], 5
    slots = [4, 0, 5, 2]
    ys = [rng.standard_normal((n + steps, layer.width)).astype(np.float32) for n in lens]
    prompt = dev(np.concatenate([y[:n] for y, n in zip(ys, lens)]))
    got = [list(np64(t)) for t in torch.split(layer(sequences(lens, slots, [1] * 4), prompt), lens)]
    seq = vbq.Sequences(4, 1, slots=dev(np.array(slots), I32))
    token = torch.zeros(4, layer.width, device=DEV)
    kept = (layer.conv_state.clone(), layer.state.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(seq, token)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = layer(seq, token)
    layer.conv_state.copy_(kept[0])
    layer.state.copy_(kept[1])
    for i in range(steps):
        token.copy_(dev(np.stack([y[n + i] for y, n in zip(ys, lens)])))
        graph.replay()
        for b, r in enumerate(np64(res)):
            got[b].append(r)
    ref = layer.reference(dev(np.concatenate(ys)), [len(y) for y in ys])
    got = np.concatenate([np.stack(g) for g in got])
    assert np.linalg.norm(got - ref) <= 0.01 * np.linalg.norm(ref)
    for b in range(4):
        assert np.linalg.norm(got[b * 3:][:3] - ref[b * 3:][:3]) <= 0.02 * np.linalg.norm(ref[b * 3:][:3])


def test_graph_replays_read_the_sequences_anew():
    """starts, slots and fresh may change between replays."""
    rng = np.random.default_rng(12)
    layer = Layer(rng, 1, 2, 64, 8)
    starts, slots, fresh = torch.zeros(4, dtype=I32, device=DEV), torch.zeros(3, dtype=I32, device=DEV), torch.ones(3, dtype=I32, device=DEV)
    seq = vbq.Sequences(3, 200, starts=starts, tokens=200, slots=slots, fresh=fresh)
    y = torch.zeros(200, layer.width, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(seq, y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = layer(seq, y)
    for lens in ([200, 0, 0], [3, 100, 97], [0, 1, 40], [65, 64, 63]):
        starts.copy_(dev(starts_of(lens), I32))
        slots.copy_(torch.randperm(8, device=DEV)[:3])
        y.copy_(dev(rng.standard_normal((200, layer.width)).astype(np.float32)))
        layer.state.fill_(float("nan"))
        layer.conv_state.fill_(float("nan"))
        graph.replay()
        n = sum(lens)
        ref = layer.reference(y[:n], [m for m in lens])
        assert np.linalg.norm(np64(res[:n]) - ref) <= 0.01 * np.linalg.norm(ref)


def test_calls_on_another_stream():
    """On a stream of their own, with the current one busy: nothing that a call makes for itself is reached by its work."""
    rng = np.random.default_rng(13)
    layer = Layer(rng, 2, 4, 128, 3)
    y = torch.randn(150, layer.width, device=DEV)
    seq = sequences([100, 49, 1], [2, 0, 1], [1, 1, 1])
    want = layer(seq, y).clone()
    side, big = torch.cuda.Stream(), torch.randn(8192, 8192, device=DEV)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        for _ in range(3):
            for _ in range(4):
                torch.mm(big, big)
            got = layer(seq, y, stream=stream)
            junk = [torch.full_like(want, JUNK) for _ in range(4)]
            side.synchronize()
            assert torch.equal(got, want)
            del junk, got
    assert vbq.vbq_device_status() is None
