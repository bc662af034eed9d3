"""Attention over caches whose memory holds more than what was appended: tokens
before a window that were never written, between the windows of rows that lie far
apart, after the last token. What no append has written must not show, whatever
bytes are there."""

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import decode_oracle as o
from test_kv_gpu import _check_attend, _held

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32 = torch.int32

# A scale of these bytes is NaN, -57000 or so, +57000 or so.
JUNK = [0xff, 0xfa, 0x7a]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


def _written(spans, kv_heads, d, junk, rng, spare=1):
    """A cache of junk bytes in which sequence b holds only the tokens of spans[b], a list of (first, end). Returns
    (cache, table, keys, values), keys and values with zeros for what was not written."""
    need = [max(e for _, e in s) // 64 + 1 + spare for s in spans]
    order = 1 + rng.permutation(sum(need)).astype(np.int32)      # page 0 is no sequence's
    table = np.zeros((len(spans), max(need)), np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    table = torch.from_numpy(table).to(DEV)
    cache = vbq.KvCache(1 + sum(need), kv_heads, d)
    cache.pages.fill_(junk)
    ks, vs = [], []
    for b, s in enumerate(spans):
        n = max(e for _, e in s)
        k, v = (np.zeros((n, kv_heads, d), np.float32) for _ in "kv")
        for i, e in s:
            k[i:e], v[i:e] = (rng.standard_normal((e - i, kv_heads, d)).astype(np.float32) for _ in "kv")
            vbq.vbq_kv_append(cache, table[b:b + 1], torch.arange(i, e, dtype=I32, device=DEV)[None],
                              torch.from_numpy(k[None, i:e]).to(DEV), torch.from_numpy(v[None, i:e]).to(DEV))
        ks.append(k)
        vs.append(v)
    return cache, table, ks, vs


@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows,heads,hk,window", [(1, 4, 2, 100), (1, 2, 2, 1), (3, 8, 2, 75), (16, 12, 2, 200), (16, 4, 4, 31)], ids=str)
def test_only_the_window_was_written(junk, d, rows, heads, hk, window):
    """The last `window` tokens of a prompt and nothing before them, at ends anywhere in a page."""
    rng = np.random.default_rng(junk + d + rows + window)
    ends = [300, 321, 383, 384, 5000]
    cache, table, ks, vs = _written([[(n - rows + 1 - window, n)] for n in ends], hk, d, junk, rng)
    pos = np.array([[n - rows + t for t in range(rows)] for n in ends], np.int32)
    _check_attend(cache, table, ks, vs, pos, heads, rng, window=window)


@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_nothing_between_the_windows_of_distant_rows(junk, d):
    rng = np.random.default_rng(junk + d)
    cache, table, ks, vs = _written([[(31, 101), (4931, 5001)], [(0, 10), (51, 165)]], 2, d, junk, rng)
    _check_attend(cache, table, ks, vs, np.array([[100, 5000, -1], [164, 9, 120]], np.int32), 8, rng, window=70)


@pytest.mark.parametrize("junk", JUNK)
def test_only_the_window_of_many_short_sequences(junk):
    """More segments than blocks: teams of warps."""
    rng = np.random.default_rng(junk)
    ends = [int(n) for n in rng.integers(90, 700, 230)]
    cache, table, ks, vs = _written([[(n - 80, n)] for n in ends], 2, 64, junk, rng)
    _check_attend(cache, table, ks, vs, np.array([[n - 1] for n in ends], np.int32), 4, rng, window=80)


def _expect_range():
    with pytest.raises(vbq.VbqError) as e:
        vbq.vbq_device_status()
    assert e.value.name == "VBQ_ERR_RANGE"


def _row_ok(out, q, row, k, v, p, scale, window=0):
    """Row `row` of the first sequence within the bound of the oracle's, at position p."""
    kd, ksc = _held(k)
    vd, vsc = _held(v)
    ref, spread, reach = o.attend(q[0, row:row + 1].float().cpu().numpy(), kd, vd, [p], scale, window, ksc)
    got = out[0, row:row + 1].float().cpu().numpy().astype(np.float64)
    return bool(o.attend_within_bound(got, ref, spread, reach, 8 * float(vsc.max()), len(k)).all())


@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 40])
def test_a_position_outside_leaves_the_sequence_s_other_rows_alone(junk, d, window):
    """The table ends in pages that hold nothing; one row's position lies past them."""
    rng = np.random.default_rng(junk + d + window)
    cache, table, ks, vs = _written([[(0, 152)]], 2, d, junk, rng, spare=2)
    q = torch.from_numpy(rng.standard_normal((1, 4, 4, d)).astype(np.float32)).to(DEV).to(torch.bfloat16)
    for far in (1 << 20, table.shape[1] * 64, 0x7fffffff):
        pos = [150, far, 151, 20]
        out = vbq.vbq_kv_attend(cache, table, torch.tensor([pos], dtype=I32, device=DEV), q, window=window)
        _expect_range()
        assert all(_row_ok(out, q, r, ks[0], vs[0], pos[r], d ** -0.5, window) for r in (0, 2, 3))


@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("entry", [-1, 1 << 30])
def test_a_page_outside_leaves_the_rows_before_it_alone(junk, d, entry):
    """One page of a sequence is outside the cache; rows that end before it are served."""
    rng = np.random.default_rng(junk + d)
    cache, table, ks, vs = _written([[(0, 200)]], 2, d, junk, rng)
    table[0, 1] = entry
    q = torch.from_numpy(rng.standard_normal((1, 3, 4, d)).astype(np.float32)).to(DEV).to(torch.bfloat16)
    pos = [10, 199, 63]
    out = vbq.vbq_kv_attend(cache, table, torch.tensor([pos], dtype=I32, device=DEV), q)
    _expect_range()
    assert all(_row_ok(out, q, r, ks[0], vs[0], pos[r], d ** -0.5) for r in (0, 2))


@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_pages_between_the_windows_of_distant_rows_may_be_gone(junk, d):
    """A table whose pages between two windows have been given back: nothing to report, nothing lost."""
    rng = np.random.default_rng(junk + d)
    cache, table, ks, vs = _written([[(31, 101), (4931, 5001)]], 2, d, junk, rng)
    table[0, 2:77] = -1
    _check_attend(cache, table, ks, vs, np.array([[100, 5000, -1]], np.int32), 8, rng, window=70)
    table[0, 77] = -1                                             # tokens 4928 ..: needed
    vbq.vbq_kv_attend(cache, table, torch.tensor([[100, 5000]], dtype=I32, device=DEV), torch.zeros(1, 2, 8, d, dtype=torch.bfloat16, device=DEV),
                      window=70)
    _expect_range()


def test_unused_rows_by_any_negative_position():
    rng = np.random.default_rng(7)
    cache, table, ks, vs = _written([[(0, 400)]], 2, 128, 0xff, rng)
    for window in (0, 90):
        got = _check_attend(cache, table, ks, vs, np.array([[399, -1, -2 ** 31, 398, -5]], np.int64), 4, rng, window=window)
        assert not got[0, [1, 2, 4]].any() and got[0, [0, 3]].all(-1).all()
