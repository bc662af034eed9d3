"""What digits the results of the gated delta rule keep: outputs and states of every
path are fp32 sums, whatever a call's sequences are, rounded once."""

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import delta_oracle as o
from test_delta_gpu import BF16, DEV, F32, I32, Layer, check_delta, dev, inputs, np64, sequences

pytestmark = pytest.mark.gpu

A = 1.0 + 2.0 ** -12                                              # lost where 11 bits are kept


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


# Sums of a terms of A and a of -1, times u: a 2^-12 u is left. Nothing but one kind of operand has more than 8 bits.
# Batch and heads so that a block takes 32 columns of a state, or 64.
@pytest.mark.parametrize("batch,heads,dv", [(1, 1, 64), (5, 16, 128)], ids=["narrow", "wide"])
@pytest.mark.parametrize("dk", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [20, 64, 70], ids=lambda n: f"{n}rows")
@pytest.mark.parametrize("what", ["state", "scores", "corrections", "queries"])
def test_outputs_keep_what_cancels(what, rows, dtype, dk, batch, heads, dv):
    """Derived: products of pairs of FP16 parts, or fp32, in sums of 2 a magnitudes of u: 2^-17 of 2 a u covers parts and sums
    (2^-22 an operand, 2^-23 a step of the tensor cores), and half a step of BF16 of the result. What an operand of 11 bits
    loses is the result itself, a 2^-12 u."""
    if what == "queries" and dtype == BF16:
        pytest.skip("BF16 queries have 8 bits")
    q, k = np.zeros((rows, dk)), np.zeros((rows, dk))
    v, b = np.zeros((rows, dv)), np.zeros(rows)
    s = np.zeros((dk, dv))
    half = dk // 2
    n = min(rows, 64, half) // 2 * 2                              # tokens whose keys the last query looks at
    t0 = rows - n                                                 # all in the last chunk, or (70 rows) in two
    if what == "state":                                           # nothing is learnt; q.S of the last row
        s[:half], s[half:] = A, 1.0
        q[:, :half], q[:, half:] = 1.0, -1.0
        a, u = half, 1.0
    else:
        sign = np.where(np.arange(n) % 2 == 0, 1.0, -1.0)
        a, u = n // 2, 0.5
        b[t0:] = 0.5
        for j in range(n):                                        # keys without a common dimension: U = beta v exactly
            k[t0 + j, 2 * j] = 1.0
            q[-1, 2 * j] = sign[j]
            v[t0 + j] = 1.0
            if what == "scores":
                q[-1, 2 * j + 1] = sign[j] * 2.0 ** -12
                k[t0 + j, 2 * j + 1] = float(sign[j] > 0)
            elif what == "corrections" and sign[j] > 0:
                b[t0 + j] = 0.5 * A
            elif what == "queries" and sign[j] > 0:
                q[-1, 2 * j] = A
    rep = lambda x, t=F32: dev(np.repeat(np.tile(x, (batch, 1))[:, None], heads, 1).astype(np.float32), t)  # noqa: E731
    gate = lambda x: dev(np.repeat(np.tile(x, batch)[:, None], heads, 1).astype(np.float32))  # noqa: E731
    state = dev(np.ascontiguousarray(np.broadcast_to(s, (batch, heads, dk, dv)), np.float32))
    got = vbq.vbq_delta_rule(vbq.Sequences(batch, rows), state, rep(q, dtype), rep(k, dtype), rep(v, dtype), gate(np.zeros(rows)), gate(b), scale=1.0,
                             normalize=False)
    got, want = np64(got).reshape(batch, rows, heads, dv)[:, -1], a * 2.0 ** -12 * u
    assert np.abs(got - want).max() <= 2.0 ** -17 * 2 * a * u + 2.0 ** -8 * want


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 128), (128, 64)], ids=str)
def test_states_of_each_sequence(dk, dv, dtype):
    """The state of every sequence by itself, short and long: fp32 sums of what contracts (2^-17 of its norm), nothing of it
    hidden behind longer sequences' or unused slots. Outputs of the same call to their bounds."""
    rng = np.random.default_rng(dk + dv)
    lens, hk, h = [1, 5, 22, 23, 28, 29, 64, 90, 200, 2], 1, 2
    q, k, v, a, b, a_log, dt = inputs(rng, sum(lens), hk, h, dk, dv, dtype, True)
    slots = rng.permutation(len(lens)).astype(np.int32)
    state = dev(rng.standard_normal((len(lens), h, dk, dv)).astype(np.float32))
    before = state.clone()
    out = vbq.vbq_delta_rule(sequences(lens, slots), state, q, k, v, a, b, a_log=dev(a_log), dt_bias=dev(dt))
    at = 0
    for n, slot in zip(lens, slots):
        s = slice(at, at + n)
        check_delta(out[s], state[slot:slot + 1], before[slot:slot + 1], [n], [0], [0], 0, q[s], k[s], v[s], a[s], b[s], a_log, dt, dk ** -0.5)
        at += n


def test_layer_tokens_of_each_sequence():
    """A layer's prompts and then single tokens, each sequence's outputs by themselves: three roundings to BF16 (2^-9 each,
    independent) are in the reference too and now and then fall the other way; 2% of the norm."""
    rng = np.random.default_rng(21)
    layer, lens, steps = Layer(rng, 2, 4, 64, 6), [70, 1, 130, 9], 5
    slots = [4, 0, 5, 2]
    ys = [rng.standard_normal((n + steps, layer.width)).astype(np.float32) for n in lens]
    got = [list(np64(t)) for t in torch.split(layer(sequences(lens, slots, [1] * 4), dev(np.concatenate([y[:n] for y, n in zip(ys, lens)]))), lens)]
    seq = vbq.Sequences(4, 1, slots=dev(np.array(slots), I32))
    for i in range(steps):
        for s, r in enumerate(np64(layer(seq, dev(np.stack([y[n + i] for y, n in zip(ys, lens)]))))):
            got[s].append(r)
    for s, y in enumerate(ys):
        ref = layer.reference(torch.from_numpy(y).to(DEV), [len(y)])
        rows = np.stack(got[s])
        for part in (slice(0, lens[s]), slice(lens[s], None)):
            assert np.linalg.norm(rows[part] - ref[part]) <= 0.02 * np.linalg.norm(ref[part])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("dk", [64, 128])
@pytest.mark.parametrize("size", [1e14, 1e-14], ids=str)
def test_keys_of_all_sizes_beside_each_other(size, dk, dtype):
    """Unit length takes a key's and a query's size away, whatever its neighbours' are: single tokens 1e14 times as large, or
    as small, as those of the same chunk (their smallness counts: 1e-14 squared is nothing beside the epsilon)."""
    rng = np.random.default_rng(dk)
    rows, h, dv = 90, 2, 64
    q, k, v, a, b, _, _ = inputs(rng, rows, h, h, dk, dv, dtype, False)
    q, k = q.clone(), k.clone()
    for t in (1, 17, 48, 70):
        k[t] = (k[t].float() * size).to(dtype)
        q[t + 3] = (q[t + 3].float() * size).to(dtype)
    state = torch.randn(1, h, dk, dv, device=DEV)
    before = state.clone()
    out = vbq.vbq_delta_rule(vbq.Sequences(1, rows), state, q, k, v, a, b)
    check_delta(out, state, before, [rows], [0], [0], 0, q, k, v, a, b, None, None, dk ** -0.5)


def test_a_large_key_leaves_earlier_tokens_alone():
    """Bit for bit: a key that comes later, as large as they get, has no say in what is computed before it."""
    rng = np.random.default_rng(5)
    for dk, at in ((64, 48), (128, 24), (64, 63)):
        q, k, v, a, b, _, _ = inputs(rng, 64, 1, 1, dk, 64, BF16, False)
        k, state = k.clone(), torch.randn(1, 1, dk, 64, device=DEV)
        run = lambda: vbq.vbq_delta_rule(vbq.Sequences(1, 64), state.clone(), q, k, v, a, b)  # noqa: E731
        want = run()
        k[at] *= 2.0 ** 46
        assert torch.equal(run()[:at], want[:at])


@pytest.mark.parametrize("batch", [1, 2])
@pytest.mark.parametrize("rows", [1, 5, 22])
def test_few_rows_in_a_call_that_may_have_many(rows, batch):
    """One place of a captured step: `rows` says 200, starts say fewer. Up to 22 rows a sequence's keys may be of any sizes:
    here |k_i| |k_j| beta is 100 between tokens while beta |k|^2 stays within 0..2."""
    rng = np.random.default_rng(rows)
    h, d = 2, 128
    lens = [rows] * batch
    q, k, v, a, b, _, _ = inputs(rng, rows * batch, h, h, d, d, BF16, False)
    k, b = k.clone(), b.clone()
    k[:], b[:] = 0, 1.0
    k[:, :, 0] = 1.0
    k[:, :, 1:9] = 0.25 * torch.randn(rows * batch, h, 8, device=DEV).to(BF16)
    for i in range(batch):
        k[i * rows], b[i * rows] = 0, 1e-4
        k[i * rows, :, 0] = 100.0
    state = torch.randn(batch, h, d, d, device=DEV)
    before = state.clone()
    seq = sequences(lens, list(range(batch)), rows=200)
    out = vbq.vbq_delta_rule(seq, state, q, k, v, a, b, normalize=False)
    check_delta(out, state, before, lens, list(range(batch)), [0] * batch, 0, q, k, v, a, b, None, None, d ** -0.5, normalize=False)
