"""The 4-bit key-value cache (vbq_kv_append, vbq_kv_read, vbq_kv_attend, through
the C ABI) against the fp64 oracle.

What the cache holds must match bit by bit: scales and codes are exact
functions of the fp32 values. Attention must be within the bound
oracle.decode_oracle.attend_within_bound derives from the kernel's roundings,
with the oracle given the cache's own (dequantised) keys and values."""

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import decode_oracle as o

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


def _table(lens, rng, spare=3, slack=1):
    """Shuffled pages for sequences of these lengths; unused entries point outside the cache."""
    need = [-(-max(n, 1) // 64) for n in lens]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    t = np.full((len(lens), max(need) + slack), 1 << 30, np.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(t).to(DEV), pages


def _fill(lens, kv_heads, d, rng, kscale=1.0, vscale=1.0):
    """A cache holding random keys and values; its memory starts as 0xff bytes
    (NaN scales), so anything read that was not written shows."""
    table, pages = _table(lens, rng)
    cache = vbq.KvCache(pages, kv_heads, d)
    cache.pages.fill_(0xff)
    ks, vs = [], []
    for b, n in enumerate(lens):
        k = (rng.standard_normal((n, kv_heads, d)) * kscale).astype(np.float32)
        v = (rng.standard_normal((n, kv_heads, d)) * vscale).astype(np.float32)
        ks.append(k)
        vs.append(v)
        if n:
            pos = torch.arange(n, dtype=I32, device=DEV)[None]
            vbq.vbq_kv_append(cache, table[b:b + 1], pos, torch.from_numpy(k).to(DEV)[None], torch.from_numpy(v).to(DEV)[None])
    return cache, table, ks, vs


def _held(x):
    q, s = o.kv_quantise(x)
    return o.kv_values(q, s), s


def _check_attend(cache, table, ks, vs, pos, heads, rng, window=0, scale=None, q=None, run=None):
    b, rows = pos.shape
    d = cache.head_dim
    if q is None:
        q = rng.standard_normal((b, rows, heads, d)) * 1.5
    qt = torch.from_numpy(np.asarray(q, np.float32)).to(DEV).to(torch.bfloat16)
    scale = d ** -0.5 if scale is None else scale
    pt = torch.from_numpy(np.asarray(pos, np.int32)).to(DEV)
    ws = vbq.vbq_kv_workspace(cache, b, rows, heads)
    out = torch.full_like(qt, float("nan"))
    (run or (lambda f: f()))(lambda: vbq.vbq_kv_attend(cache, table, pt, qt, scale=scale, window=window, out=out, workspace=ws))
    torch.cuda.synchronize()
    got = out.float().cpu().numpy().astype(np.float64)
    qd = qt.float().cpu().numpy()
    again = torch.full_like(qt, float("nan"))
    vbq.vbq_kv_attend(cache, table, pt, qt, scale=scale, window=window, out=again, workspace=ws)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)), "a repeated call differs"
    for i in range(b):
        n = ks[i].shape[0]
        k, kscales = _held(ks[i]) if n else (np.zeros((0, cache.kv_heads, d)), np.zeros((0, cache.kv_heads, d // 64), np.float16))
        v, vscales = _held(vs[i]) if n else (k, kscales)
        ref, spread, reach = o.attend(qd[i], k, v, pos[i], scale, window, kscales)
        ok = o.attend_within_bound(got[i], ref, spread, reach, 8 * float(vscales.max(initial=0)), n)
        assert ok.all(), f"sequence {i}: {int((~ok).sum())} of {ok.size} outputs outside the bound, worst " \
                         f"{np.abs(got[i] - ref)[~ok].max()}"
    assert vbq.vbq_device_status() is None
    return got


# ---------------------------------------------------------------------------
# append and read
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rot", ["none", "part", "all"])
def test_append_matches_oracle(d, dtype, rot):
    rng = np.random.default_rng(hash((d, str(dtype), rot)) % 1000)
    lens, rows, heads, hk = [130, 67, 64], 3, 6, 3
    table, pages = _table(lens, rng)
    cache = vbq.KvCache(pages, hk, d)
    cache.pages.fill_(0xff)
    fused = torch.from_numpy(rng.standard_normal((3, rows, heads + 2 * hk, d)).astype(np.float32)).to(DEV).to(dtype)
    pos = np.array([[127, 129, 3], [66, -1, 0], [63, 62, 5]], np.int32)
    r = {"none": 0, "part": 32, "all": d}[rot]
    cos = sin = None
    if r:
        angle = rng.uniform(-9, 9, (130, r // 2))
        cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    ct, st = (None if a is None else torch.from_numpy(a).to(DEV) for a in (cos, sin))
    pt = torch.from_numpy(pos).to(DEV)
    q_out = vbq.vbq_kv_append(cache, table, pt, fused[:, :, heads:heads + hk], fused[:, :, heads + hk:], q=fused[:, :, :heads],
                              cos=ct, sin=st)
    kr, vr = vbq.vbq_kv_read(cache, table, pt)
    torch.cuda.synchronize()
    x = fused.float().cpu().numpy().reshape(-1, heads + 2 * hk, d)
    flat = pos.reshape(-1)
    if r:
        at = np.maximum(flat, 0)
        x[:, :heads + hk] = o.rotate(x[:, :heads + hk], cos[at], sin[at])
    live = flat >= 0
    kq = np.where(live[:, None, None], _held(x[:, heads:heads + hk])[0], 0.0)
    vq = np.where(live[:, None, None], _held(x[:, heads + hk:])[0], 0.0)
    assert np.array_equal(kr.cpu().numpy().reshape(kq.shape), kq.astype(np.float32))
    assert np.array_equal(vr.cpu().numpy().reshape(vq.shape), vq.astype(np.float32))
    want = torch.from_numpy(np.where(live[:, None, None], x[:, :heads], 0.0).astype(np.float32)).to(torch.bfloat16)
    assert torch.equal(q_out.cpu().reshape(want.shape), want)
    assert vbq.vbq_device_status() is None


def test_append_ties_and_extremes_match_oracle():
    """Quotients on and an ulp beside half-integers, scale midpoints, zeros, subnormal scales, infinities, NaN."""
    rng = np.random.default_rng(11)
    n = 640
    x = rng.standard_normal((n, 1, 64)).astype(np.float32)
    s = np.float32(2.0) ** rng.integers(-24, 15, n).astype(np.float32) * rng.integers(1, 2, n)
    s = (s * (1 + rng.integers(0, 1024, n) / 1024)).astype(np.float16).astype(np.float32)
    for i in range(n):
        if i % 4 == 0:
            continue
        x[i, 0, 0] = 7 * s[i]                                     # the scale is s[i]
        half = (rng.integers(0, 7, 63) + np.float32(0.5)) * s[i] * rng.choice([-1, 1], 63)
        nudge = [0, 1, -1][i % 4 - 1]
        x[i, 0, 1:] = half if nudge == 0 else np.nextafter(half, np.float32(nudge * np.inf) * np.sign(half), dtype=np.float32)
    h = np.arange(1, 64, dtype=np.uint16) * 997 % 31000 + 1       # maxima on and beside FP16 midpoints times 7
    mid = 3.5 * (h.view(np.float16).astype(np.float64) + (h + 1).astype(np.uint16).view(np.float16).astype(np.float64))
    for j, m in enumerate(mid.astype(np.float32)):
        x[4 * j, 0] = np.clip(x[4 * j, 0], -0.1, 0.1) * m
        x[4 * j, 0, 9] = [m, np.nextafter(m, np.float32(np.inf)), np.nextafter(m, np.float32(0))][j % 3]
    x[4 * 70, 0] = 0.0
    x[4 * 71, 0] = 1e-9
    x[4 * 72, 0, 3] = np.inf
    x[4 * 73, 0, 3] = -np.inf
    x[4 * 74, 0, 5] = np.nan
    x[4 * 75, 0] = np.nan
    x[4 * 76, 0] = 3e38
    x[4 * 77, 0, 2] = 458633.0                                    # just above 7 * 65519
    x[4 * 78, 0] = -0.0
    table, pages = _table([n], rng)
    cache = vbq.KvCache(pages, 1, 64)
    xt = torch.from_numpy(x).to(DEV)[None]
    pos = torch.from_numpy(rng.permutation(n).astype(np.int32)).to(DEV)[None]
    vbq.vbq_kv_append(cache, table, pos, xt, -xt)
    k, v = vbq.vbq_kv_read(cache, table, pos)
    want = _held(x)[0].astype(np.float32)
    assert np.array_equal(k[0].cpu().numpy(), want)
    assert np.array_equal(v[0].cpu().numpy(), -want)


def test_append_leaves_other_tokens_alone():
    rng = np.random.default_rng(12)
    cache, table, ks, vs = _fill([100], 2, 128, rng)
    before = [t.clone() for t in vbq.vbq_kv_read(cache, table, torch.arange(100, dtype=I32, device=DEV)[None])]
    k = torch.randn(1, 2, 2, 128, device=DEV)
    vbq.vbq_kv_append(cache, table, torch.tensor([[17, 64]], dtype=I32, device=DEV), k, k)
    after = vbq.vbq_kv_read(cache, table, torch.arange(100, dtype=I32, device=DEV)[None])
    for x, y in zip(before, after):
        same = (x == y).all(-1).all(-1)[0].cpu().numpy()
        assert np.flatnonzero(~same).tolist() == [17, 64]


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,hk", [(4, 4), (8, 2), (9, 1), (24, 2), (5, 1)], ids=lambda x: str(x))
def test_attend_lengths(d, heads, hk):
    rng = np.random.default_rng(d + heads)
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 128, 200, 0]
    cache, table, ks, vs = _fill(lens, hk, d, rng)
    pos = np.array([[n - 1] for n in lens], np.int32)
    _check_attend(cache, table, ks, vs, pos, heads, rng)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows,heads,hk", [(2, 4, 4), (5, 8, 2), (16, 4, 1), (16, 20, 1), (7, 3, 3), (16, 64, 1)], ids=lambda x: str(x))
@pytest.mark.parametrize("window", [0, 1, 17, 100])
def test_attend_chunks(d, rows, heads, hk, window):
    """Several rows per sequence, causal among themselves, some unused, one sequence wholly unused."""
    rng = np.random.default_rng(rows * heads + window)
    lens = [rows, 90, 300, 129, 80]
    cache, table, ks, vs = _fill(lens, hk, d, rng)
    pos = np.array([[n - rows + t for t in range(rows)] for n in lens], np.int32)
    pos[1, rows // 2] = -1
    pos[2] = pos[2, ::-1]                                         # any order
    pos[3, 0] = 0                                                 # far from the others
    pos[4] = -1
    _check_attend(cache, table, ks, vs, pos, heads, rng, window=window)


@pytest.mark.parametrize("d,heads,hk,lens,rows,window", [
    (128, 8, 2, [20000], 1, 0), (64, 4, 4, [9000, 3, 0, 4097], 1, 0), (128, 16, 2, [5000, 700], 4, 3000),
    (256, 3, 1, [6000], 2, 0), (128, 4, 4, [1500] * 40, 1, 0)], ids=str)
def test_attend_long(d, heads, hk, lens, rows, window):
    rng = np.random.default_rng(len(lens) + d)
    cache, table, ks, vs = _fill(lens, hk, d, rng)
    pos = np.array([[max(n - rows, -1) + t if n else -1 for t in range(rows)] for n in lens], np.int32)
    pos = np.minimum(pos, np.array(lens)[:, None] - 1)
    _check_attend(cache, table, ks, vs, pos, heads, rng, window=window)


@pytest.mark.parametrize("kscale,vscale,qscale", [(1e-4, 1e-4, 1.0), (50.0, 1e4, 1.0), (1.0, 1.0, 2.0 ** -60), (3e-3, 1.0, 2.0 ** 9)])
def test_attend_magnitudes(kscale, vscale, qscale):
    rng = np.random.default_rng(21)
    cache, table, ks, vs = _fill([333], 2, 128, rng, kscale, vscale)
    _check_attend(cache, table, ks, vs, np.array([[332]]), 4, rng, q=rng.standard_normal((1, 1, 4, 128)) * qscale)


def test_attend_mixed_value_scales():
    """Value scales across the whole FP16 range in one sequence, growing and shrinking; groups of zeros."""
    rng = np.random.default_rng(22)
    n = 500
    cache, table, _, _ = _fill([n], 1, 128, rng)
    k = rng.standard_normal((n, 1, 128)).astype(np.float32)
    v = (rng.standard_normal((n, 1, 128)) * 10.0 ** rng.uniform(-6, 5, (n, 1, 1))).astype(np.float32)
    v[5:9], v[100, :, :64] = 0, 0
    pos = torch.arange(n, dtype=I32, device=DEV)[None]
    vbq.vbq_kv_append(cache, table, pos, torch.from_numpy(k).to(DEV)[None], torch.from_numpy(v).to(DEV)[None])
    for p in (0, 63, 64, 200, n - 1):
        _check_attend(cache, table, [k], [v], np.array([[p]]), 2, rng)


def test_attend_peaked_and_zero_scores():
    rng = np.random.default_rng(23)
    cache, table, ks, vs = _fill([400], 1, 64, rng, kscale=20.0)
    _check_attend(cache, table, ks, vs, np.array([[399]]), 8, rng, q=rng.standard_normal((1, 1, 8, 64)) * 40)
    _check_attend(cache, table, ks, vs, np.array([[399]]), 8, rng, q=np.zeros((1, 1, 8, 64)))
    _check_attend(cache, table, ks, vs, np.array([[399]]), 8, rng, scale=0.0)
    _check_attend(cache, table, ks, vs, np.array([[399]]), 8, rng, scale=-0.3)


def test_attend_stays_within_rows_of_nan_queries():
    """A row of NaN queries leaves the other rows' results alone."""
    rng = np.random.default_rng(24)
    cache, table, ks, vs = _fill([200], 2, 128, rng)
    q = torch.randn(1, 3, 4, 128, device=DEV).to(torch.bfloat16)
    pos = torch.tensor([[197, 198, 199]], dtype=I32, device=DEV)
    want = vbq.vbq_kv_attend(cache, table, pos, q)
    q[0, 1, 2] = float("nan")
    got = vbq.vbq_kv_attend(cache, table, pos, q)
    same = (got == want).all(-1)[0]
    assert not same[1, 2] and int((~same).sum()) == 1


def test_attend_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(25)
    cache, table, ks, vs = _fill([700, 90], 2, 128, rng)
    pos = np.array([[699], [89]], np.int32)
    side = torch.cuda.Stream()

    def on_side(f):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            f()
        torch.cuda.current_stream().wait_stream(side)

    def in_graph(f):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        for _ in range(3):
            g.replay()

    _check_attend(cache, table, ks, vs, pos, 8, rng, run=on_side)
    _check_attend(cache, table, ks, vs, pos, 8, rng, run=in_graph)


def test_attend_follows_append_in_stream_order():
    """Append and attend one token at a time, as a decode loop does, without waiting in between."""
    rng = np.random.default_rng(26)
    n, hk, heads, d = 150, 2, 4, 64
    table, pages = _table([n], rng)
    cache = vbq.KvCache(pages, hk, d)
    cache.pages.fill_(0xff)
    k, v = (rng.standard_normal((n, hk, d)).astype(np.float32) for _ in "kv")
    kt, vt = torch.from_numpy(k).to(DEV), torch.from_numpy(v).to(DEV)
    q = torch.randn(n, 1, 1, heads, d, device=DEV).to(torch.bfloat16)
    pos = torch.arange(n, dtype=I32, device=DEV).reshape(n, 1, 1)
    ws = vbq.vbq_kv_workspace(cache, 1, 1, heads)
    outs = torch.empty_like(q)
    for i in range(n):
        vbq.vbq_kv_append(cache, table, pos[i], kt[None, i:i + 1], vt[None, i:i + 1])
        vbq.vbq_kv_attend(cache, table, pos[i], q[i], out=outs[i], workspace=ws)
    kd, ksc = _held(k)
    vd, vsc = _held(v)
    ref, spread, reach = o.attend(q[:, 0, 0].float().cpu().numpy(), kd, vd, np.arange(n), d ** -0.5, 0, ksc)
    ok = o.attend_within_bound(outs[:, 0, 0].float().cpu().numpy(), ref, spread, reach, 8 * float(vsc.max()), n)
    assert ok.all()


def test_workspace_serves_smaller_calls():
    rng = np.random.default_rng(27)
    cache, table, ks, vs = _fill([3000, 100, 900], 2, 128, rng)
    ws = vbq.vbq_kv_workspace(cache, 3, 8, 16)
    pos = torch.tensor([[2999], [99], [899]], dtype=I32, device=DEV)
    for heads, rows, b in ((16, 1, 3), (2, 8, 1), (4, 1, 2), (16, 8, 3), (8, 2, 2)):
        q = torch.randn(b, rows, heads, 128, device=DEV).to(torch.bfloat16)
        p = (pos[:b] - torch.arange(rows, dtype=I32, device=DEV)).contiguous()
        x = vbq.vbq_kv_attend(cache, table[:b], p, q, workspace=ws)
        y = vbq.vbq_kv_attend(cache, table[:b], p, q)
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_pages_past_four_gigabytes():
    d, hk = 128, 8
    per = vbq.vbq_kv_page_bytes(hk, d)
    pages = (5 << 30) // per
    cache = vbq.KvCache(pages, hk, d)
    rng = np.random.default_rng(28)
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=I32, device=DEV)
    k, v = (rng.standard_normal((150, hk, d)).astype(np.float32) for _ in "kv")
    pos = torch.arange(150, dtype=I32, device=DEV)[None]
    vbq.vbq_kv_append(cache, table, pos, torch.from_numpy(k).to(DEV)[None], torch.from_numpy(v).to(DEV)[None])
    assert np.array_equal(vbq.vbq_kv_read(cache, table, pos)[0][0].cpu().numpy(), _held(k)[0].astype(np.float32))
    _check_attend(cache, table, [k], [v], np.array([[149]]), 16, rng)


def test_positions_and_pages_outside_the_cache_are_reported():
    """They are skipped by the kernels' own checks and reported by vbq_device_status; other rows are served."""
    rng = np.random.default_rng(29)
    cache, table, ks, vs = _fill([100, 100], 1, 64, rng)
    x = torch.randn(2, 1, 1, 64, device=DEV)
    before = cache.pages.clone()
    for pos, entry in (([[1 << 20], [-1]], None), ([[5], [-1]], 1 << 20), ([[5], [-1]], -7)):
        t = table.clone()
        if entry is not None:
            t[0, 0] = entry
        p = torch.tensor(pos, dtype=I32, device=DEV)
        vbq.vbq_kv_append(cache, t, p, x, x)
        with pytest.raises(vbq.VbqError) as e:
            vbq.vbq_device_status()
        assert e.value.name == "VBQ_ERR_RANGE" and torch.equal(before, cache.pages)
        k, _ = vbq.vbq_kv_read(cache, t, p)
        assert not k.any()
        with pytest.raises(vbq.VbqError):
            vbq.vbq_device_status()
        q = torch.randn(2, 1, 2, 64, device=DEV).to(torch.bfloat16)
        p[1] = 99
        out = vbq.vbq_kv_attend(cache, t, p, q)
        with pytest.raises(vbq.VbqError) as e:
            vbq.vbq_device_status()
        assert e.value.name == "VBQ_ERR_RANGE"
        assert torch.equal(out[1:], vbq.vbq_kv_attend(cache, table[1:], p[1:].contiguous(), q[1:].contiguous()))
        vbq.vbq_device_status()
    cos = torch.ones(4, 16, device=DEV)
    vbq.vbq_kv_append(cache, table, torch.tensor([[4], [3]], dtype=I32, device=DEV), x, x, cos=cos, sin=cos)
    with pytest.raises(vbq.VbqError):
        vbq.vbq_device_status()


@pytest.mark.parametrize("batch,hk,heads,rows,most", [(1024, 1, 2, 1, 200), (300, 2, 6, 3, 150), (1024, 3, 3, 2, 40)])
def test_attend_many_sequences(batch, hk, heads, rows, most):
    """More segments than blocks, short and uneven, some empty; every output checked on a sample of sequences."""
    rng = np.random.default_rng(batch + rows)
    lens = [int(n) for n in rng.integers(0, most, batch)]
    table, pages = _table(lens, rng)
    cache = vbq.KvCache(pages, hk, 64)
    cache.pages.fill_(0xff)
    n = max(lens)
    k, v = (rng.standard_normal((batch, n, hk, 64)).astype(np.float32) for _ in "kv")
    pos = np.where(np.arange(n)[None] < np.array(lens)[:, None], np.arange(n)[None], -1).astype(np.int32)
    vbq.vbq_kv_append(cache, table, torch.from_numpy(pos).to(DEV), torch.from_numpy(k).to(DEV), torch.from_numpy(v).to(DEV))
    q = torch.randn(batch, rows, heads, 64, device=DEV).to(torch.bfloat16)
    at = np.array([[m - rows + t if m else -1 for t in range(rows)] for m in lens], np.int32)
    at = np.maximum(at, -1)
    out = vbq.vbq_kv_attend(cache, table, torch.from_numpy(at).to(DEV), q).float().cpu().numpy()
    qd = q.float().cpu().numpy()
    for i in list(range(8)) + [int(x) for x in rng.integers(8, batch, 60)] + [batch - 1]:
        m = lens[i]
        if m == 0:
            assert not out[i].any()
            continue
        kd, ks = _held(k[i, :m])
        vd, vs = _held(v[i, :m])
        ref, spread, reach = o.attend(qd[i], kd, vd, at[i], 0.125, 0, ks)
        assert o.attend_within_bound(out[i], ref, spread, reach, 8 * float(vs.max()), m).all(), i
    assert vbq.vbq_device_status() is None


def test_one_workspace_serves_every_shape():
    """Head dimensions, head counts and tiles in turn on one workspace, each as with its own."""
    rng = np.random.default_rng(31)
    made = [_fill([5000, 300], hk, d, rng)[:2] for hk, d in ((2, 128), (1, 64), (2, 256), (4, 64))]
    ws = torch.zeros(max(vbq.vbq_kv_workspace_bytes(c, 2, 16, 8) for c, _ in made), dtype=torch.uint8, device=DEV)
    pos = torch.tensor([[4999], [299]], dtype=I32, device=DEV)
    for _ in range(2):
        for cache, table in made:
            for rows in (1, 16):
                q = torch.randn(2, rows, 8, cache.head_dim, device=DEV).to(torch.bfloat16)
                p = (pos - torch.arange(rows, dtype=I32, device=DEV)).contiguous()
                x, y = vbq.vbq_kv_attend(cache, table, p, q, workspace=ws), vbq.vbq_kv_attend(cache, table, p, q)
                assert torch.equal(x.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("d,rows,heads,hk", [(64, 1, 6, 6), (64, 3, 12, 3), (128, 1, 16, 8), (128, 5, 9, 3), (256, 1, 8, 4),
                                             (256, 3, 8, 2)], ids=str)
@pytest.mark.parametrize("lens", ["short", "equal", "uneven", "one_long"])
@pytest.mark.parametrize("window", [0, 90])
def test_attend_segments_by_teams(d, rows, heads, hk, lens, window):
    """More segments than blocks: by one warp, by a few, by all of a block's, and as a list that is cut."""
    rng = np.random.default_rng(d + rows + len(lens) + window)
    n = 460 // hk                                                 # sequences
    if lens == "short":
        lens = [int(x) for x in rng.integers(0, 70, n)]
    elif lens == "equal":
        lens = [330] * n
    elif lens == "uneven":
        lens = [int(x) for x in np.exp(rng.uniform(0, np.log(1500), n))]
    else:
        lens = [int(x) for x in rng.integers(1, 130, n)]
        lens[n // 2] = 9000
    cache, table, ks, vs = _fill(lens, hk, d, rng)
    pos = np.array([[max(m - rows + t, -1) if m else -1 for t in range(rows)] for m in lens], np.int32)
    pos[n // 3, 0] = -1
    _check_attend(cache, table, ks, vs, pos, heads, rng, window=window)


def test_attend_teams_report_pages_outside_the_cache():
    """One sequence's page is outside: reported, and every other sequence has what it has without."""
    rng = np.random.default_rng(33)
    cache, table, ks, vs = _fill([200] * 100, 3, 128, rng)
    pos = torch.full((100, 1), 199, dtype=I32, device=DEV)
    q = torch.randn(100, 1, 6, 128, device=DEV).to(torch.bfloat16)
    want = vbq.vbq_kv_attend(cache, table, pos, q)
    assert vbq.vbq_device_status() is None
    table[41, 2] = -3
    got = vbq.vbq_kv_attend(cache, table, pos, q)
    with pytest.raises(vbq.VbqError) as e:
        vbq.vbq_device_status()
    assert e.value.name == "VBQ_ERR_RANGE"
    same = (got == want).flatten(1).all(1).cpu()
    same[41] = True
    assert bool(same.all())


@pytest.mark.parametrize("d,rows,heads,hk", [(64, 1, 1, 1), (64, 3, 4, 1), (64, 1, 5, 1), (128, 1, 4, 1), (128, 5, 2, 2), (128, 1, 3, 3),
                                             (256, 1, 2, 1), (256, 2, 2, 2)], ids=str)
@pytest.mark.parametrize("window", [0, 4000])
def test_attend_many_parts_few_rows(d, rows, heads, hk, window):
    """Few segments of few rows, cut into many parts; rows far apart, so that parts hold keys of some rows only; an unused row."""
    rng = np.random.default_rng(d + 10 * rows + heads + window)
    lens = [9000, 2500]
    cache, table, ks, vs = _fill(lens, hk, d, rng)
    pos = np.array([[n - 1 - 1500 * t for t in range(rows)] for n in lens], np.int32)
    pos[1, rows // 2:] = -1 if rows > 1 else pos[1, rows // 2:]
    pos = np.maximum(pos, -1)
    _check_attend(cache, table, ks, vs, pos, heads, rng, window=window)
    _check_attend(cache, table[:1], ks[:1], vs[:1], pos[:1], heads, rng, window=window)
