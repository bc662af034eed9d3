"""The residual norm and the sampler (vbq_residual_norm, vbq_sample) against the
fp64 oracle, through the C ABI."""

import numpy as np
import pytest
import torch

import paper_2607_02893_gb300 as vbq
from oracle import decode_oracle as o

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2607_02893_gb300 import build
    build.build()
    vbq.load()
    torch.cuda.init()


def _bf16(a):
    return torch.from_numpy(a).to(torch.bfloat16).float().numpy()


# ---------------------------------------------------------------------------
# residual norm
# ---------------------------------------------------------------------------

def _norm_ok(got, ref):
    # fp32: a sum of up to 2^20 squares in a tree of chains (2^-16 relative covers it), a division, a root and two
    # products; then BF16: 2^-9, twice that allowed. Subnormal outputs: half the smallest step.
    return np.abs(got - ref) <= (2.0 ** -8 + 2.0 ** -16) * np.abs(ref) + 2.0 ** -133


@pytest.mark.parametrize("rows,width", [(1, 1), (1, 768), (3, 63), (16, 4096), (2, 4097), (5, 16384), (1, 16388), (2, 20001), (1, 70000), (300, 100)],
                         ids=lambda x: str(x))
@pytest.mark.parametrize("x_type", [torch.float32, torch.bfloat16], ids=["xf32", "xbf16"])
@pytest.mark.parametrize("r_type", [torch.float32, torch.bfloat16, None], ids=["rf32", "rbf16", "none"])
def test_norm_matches_oracle(rows, width, x_type, r_type):
    rng = np.random.default_rng(rows * width)
    x = torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).to(x_type)
    r = None if r_type is None else torch.from_numpy((rng.standard_normal((rows, width)) * 5).astype(np.float32)).to(r_type)
    w = rng.standard_normal(width).astype(np.float32)
    rd = None if r is None else r.to(DEV)
    out, new = vbq.vbq_residual_norm(x.to(DEV), rd, torch.from_numpy(w).to(DEV), 1e-5)
    ref, rr = o.residual_norm(x.float().numpy(), None if r is None else r.float().numpy(), w, 1e-5,
                              _bf16 if r_type is torch.bfloat16 else lambda a: a)
    if r is not None:
        assert np.array_equal(new.float().cpu().numpy(), rr.astype(np.float32))
        assert torch.equal(rd.cpu(), r)                           # untouched
        vbq.vbq_residual_norm(x.to(DEV), rd, torch.from_numpy(w).to(DEV), 1e-5, residual_out=rd)
        assert torch.equal(rd, new)                               # in place
    assert _norm_ok(out.float().cpu().numpy(), ref).all()


def test_norm_of_zero_rows_zeros_and_extremes():
    w = torch.ones(512, device=DEV)
    out, _ = vbq.vbq_residual_norm(torch.zeros(0, 512, device=DEV), None, w, 1e-5)
    assert out.shape == (0, 512)
    out, _ = vbq.vbq_residual_norm(torch.zeros(2, 512, device=DEV), None, w, 0.0)
    assert torch.isnan(out).all()                                 # 0 * rsqrt(0), as the formula gives
    out, _ = vbq.vbq_residual_norm(torch.zeros(2, 512, device=DEV), None, w, 1e-6)
    assert not out.any()
    x = np.full((1, 512), 1e15, np.float32)
    x[0, ::3] = -3e14
    out, _ = vbq.vbq_residual_norm(torch.from_numpy(x).to(DEV), None, w, 1e-5)
    assert _norm_ok(out.float().cpu().numpy(), o.residual_norm(x, None, np.ones(512), 1e-5, None)[0]).all()
    x = torch.randn(3, 512, device=DEV)
    want = vbq.vbq_residual_norm(x, None, w, 1e-5)[0]
    x[1, 7] = float("inf")
    got = vbq.vbq_residual_norm(x, None, w, 1e-5)[0]
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and torch.isnan(got[1, 7])


def test_norm_batch_shape_and_stream():
    x = torch.randn(2, 3, 256, device=DEV)
    w = torch.rand(256, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = vbq.vbq_residual_norm(x, None, w, 1e-5)[0]
    torch.cuda.synchronize()
    b = vbq.vbq_residual_norm(x.reshape(6, 256), None, w, 1e-5)[0]
    assert torch.equal(a.reshape(6, 256), b)


# ---------------------------------------------------------------------------
# sampler
# ---------------------------------------------------------------------------

# A decision (a cut, the draw) may go the other way where fp64 has it within this
# of its threshold, relative to the whole mass: fp32 exponents err by a few 2^-24
# times their argument (below 128 here) and whole multiples of 2^-32 by half of
# one for each of 2^18 tokens.
NEAR = 2.0 ** -14


def _params(b, **over):
    p = {"temperature": (1.0, torch.float32), "top_k": (0, torch.int32), "top_p": (1.0, torch.float32),
         "min_p": (0.0, torch.float32), "u": (0.5, torch.float32)}
    return {k: torch.as_tensor(over[k], dtype=t).expand(b).contiguous().to(DEV) if k in over else torch.full((b,), v, dtype=t, device=DEV)
            for k, (v, t) in p.items()}


def _draw(logits, **over):
    lt = torch.as_tensor(logits) if not isinstance(logits, torch.Tensor) else logits
    lt = lt.to(DEV)
    p = _params(lt.shape[0], **over)
    t, pr, k = vbq.vbq_sample(lt, p["temperature"], p["top_k"], p["top_p"], p["min_p"], p["u"])
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (t, pr, k)] + [{n: v.cpu().numpy() for n, v in p.items()}]


def _check(logits, **over):
    lt = torch.as_tensor(logits)
    tok, prob, kept, p = _draw(lt, **over)
    lf = lt.float().numpy()
    sure = 0
    for b in range(lf.shape[0]):
        e, mask, edge = o.sample_filters(lf[b], p["temperature"][b], int(p["top_k"][b]), float(p["top_p"][b]), float(p["min_p"][b]))
        total = e.sum()
        if total == 0:
            assert (tok[b], prob[b], kept[b]) == (-1, 0.0, 0)
            continue
        if edge > NEAR:
            sure += 1
            assert kept[b] == mask.sum(), f"row {b}: {kept[b]} kept, not {mask.sum()}"
        t = int(tok[b])
        assert 0 <= t < lf.shape[1]
        if edge > NEAR:
            assert mask[t], f"row {b}: token {t} was filtered out"
            upto = e[:t + 1].sum()
            want = float(p["u"][b]) * total
            assert upto - e[t] <= want + NEAR * total and upto >= want - NEAR * total, f"row {b}: token {t} is not the draw"
            assert abs(prob[b] - e[t] / total) <= 2.0 ** -16 * e[t] / total + 2.0 ** -40
    return tok, prob, kept, sure


@pytest.mark.parametrize("vocab", [1, 2, 31, 1000, 1025, 32000, 128256, 151937, 1 << 18])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_sample_matches_oracle(vocab, dtype):
    rng = np.random.default_rng(vocab)
    b = 12
    logits = torch.from_numpy((rng.standard_normal((b, vocab)) * 3).astype(np.float32)).to(dtype)
    logits[:, rng.integers(0, vocab, 5)] += 6
    logits = logits.to(dtype)
    u = torch.from_numpy(rng.random(b).astype(np.float32))
    sure = 0
    for over in ({}, {"temperature": 0.3}, {"top_k": 1}, {"top_k": 50}, {"top_k": [5, 900, 1024, 1025, 3000, 40000] * 2}, {"top_p": 0.9},
                 {"top_p": [0.05, 0.5, 0.99, 0.9999, 0.0, 1.5] * 2}, {"min_p": 0.05}, {"top_k": 40, "top_p": 0.8, "min_p": 0.02, "temperature": 1.4},
                 {"top_k": 6000, "top_p": 0.97, "temperature": 2.5}, {"top_p": 0.95, "temperature": 5.0}, {"temperature": 0.0}, {"min_p": 3.0}):
        sure += _check(logits, u=u, **over)[3]
    assert sure > 0 or vocab < 3


def test_sample_ties():
    """Equal logits, as BF16 heads give by the hundred: cuts keep the lowest indices, the draw is by index."""
    flat = torch.zeros(6, 1000)
    tok, prob, kept, _ = _check(flat, top_k=[1, 10, 999, 1000, 2000, 0], u=0.999)
    assert kept.tolist() == [1, 10, 999, 1000, 1000, 1000] and tok.tolist() == [0, 9, 998, 999, 999, 999]
    tok, _, kept, _ = _check(flat, top_p=[0.0005, 0.25, 0.5, 0.75, 0.0, -1.0], u=[0.0, 0.49, 0.51, 0.25, 0.7, 0.7])
    assert kept.tolist() == [1, 250, 500, 750, 1, 1] and tok.tolist() == [0, 122, 254, 187, 0, 0]   # fp32 0.51 is below 0.51
    two = torch.zeros(2, 131072)
    two[:, 1::2] = 1.0                                            # 65536 of each
    tok, _, kept, _ = _check(two, top_k=[65536 + 10, 7], u=0.9999)
    assert kept.tolist() == [65546, 7] and tok[1] == 13
    tok, _, kept, _ = _check(two, top_k=65536 + 1000, top_p=0.999, u=0.5)
    assert kept[0] == kept[1] > 65536
    z = torch.tensor([[0.0, -0.0, 0.0, -1.0]])
    assert _draw(z, top_k=2, u=0.9)[0][0] == 1                    # -0 ties with 0


def test_sample_infinities_and_nan():
    inf, nan = float("inf"), float("nan")
    rows = torch.tensor([[-inf, 2.0, -inf, 1.0], [-inf] * 4, [nan] * 4, [nan, 0.0, nan, -inf], [1.0, inf, 0.0, inf], [-inf, -inf, -3e38, -inf],
                         [3e38, -3e38, 3e38, 0.0]])
    tok, prob, kept, _ = _check(rows, u=0.6)
    assert tok.tolist() == [1, -1, -1, 1, 3, 2, 2] and kept.tolist() == [2, 0, 0, 1, 4, 1, 4]
    tok, prob, kept, _ = _check(rows, u=0.6, temperature=0.0)
    assert tok.tolist() == [1, -1, -1, 1, 1, 2, 0] and kept.tolist() == [1, 0, 0, 1, 1, 1, 1]
    tok, _, kept, _ = _check(rows, u=0.6, top_k=3, top_p=0.5)
    assert tok.tolist() == [1, -1, -1, 1, 1, 2, 0]
    lowest = torch.full((1, 5000), torch.finfo(torch.float32).min)
    lowest[0, 4321] = -1.0
    tok, prob, kept, _ = _check(lowest, u=0.999, top_p=0.9)
    assert tok[0] == 4321 and prob[0] == 1.0 and kept[0] == 1


def test_sample_draw_edges():
    l = torch.log(torch.tensor([[0.25, 0.25, 0.25, 0.25]]))
    for u, want in ((0.0, 0), (0.25, 1), (0.5, 2), (0.74, 2), (0.75, 3), (1 - 2.0 ** -24, 3)):
        assert _draw(l, u=u)[0][0] == want
    assert _draw(l, u=1.0)[0][0] == 3 and _draw(l, u=-1.0)[0][0] == 0 and _draw(l, u=float("nan"))[0][0] == 0
    assert _draw(l, temperature=float("nan"))[0][0] == 0 and _draw(l, temperature=-1.0)[0][0] == 0
    far = torch.zeros(1, 70000)
    far[0, 0] = 40.0                                              # the others weigh 4e-18 each: nothing
    assert _draw(far, u=1 - 2.0 ** -24)[0][0] == 0


def test_sample_frequencies():
    rng = np.random.default_rng(8)
    l = torch.from_numpy(rng.standard_normal((1, 50)).astype(np.float32)).expand(4096, 50).contiguous()
    u = (torch.arange(4096) + 0.5) / 4096
    tok, _, _, _ = _draw(l, u=u, temperature=0.7)
    e, _, _ = o.sample_filters(l[0].numpy(), np.float32(0.7), 0, 1.0, 0.0)
    assert np.abs(np.bincount(tok, minlength=50) - 4096 * e / e.sum()).max() <= 1.01


def test_sample_strided_rows_and_optional_outputs():
    x = torch.randn(3, 2000, device=DEV)
    view = x[:, 500:1501]
    p = _params(3, top_p=0.9, u=[0.1, 0.5, 0.9])
    a = vbq.vbq_sample(view, *p.values())
    b = vbq.vbq_sample(view.contiguous(), *p.values())
    assert all(torch.equal(i, j) for i, j in zip(a, b))
    t, pr, k = vbq.vbq_sample(view, *p.values(), probs=False, kept=False)
    assert pr is None and k is None and torch.equal(t, a[0])
    h = x.to(torch.bfloat16)[:, 501:1500]                         # rows that start on any element
    a, b = vbq.vbq_sample(h, *p.values()), vbq.vbq_sample(h.contiguous(), *p.values())
    assert all(torch.equal(i, j) for i, j in zip(a, b))


def test_sample_in_a_graph_repeats():
    x = torch.randn(4, 128256, device=DEV) * 3
    p = _params(4, top_k=100, top_p=0.95, u=[0.1, 0.4, 0.6, 0.9])
    want = [t.clone() for t in vbq.vbq_sample(x, *p.values())]
    got = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vbq.vbq_sample(x, *p.values(), tokens=got[0], probs=got[1], kept=got[2])
    for _ in range(20):
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(i, j) for i, j in zip(want, got))


@pytest.mark.parametrize("vocab", [3000, 20000, 128256, 1 << 18])
@pytest.mark.parametrize("spread", [0.0, 1e-7, 1e-3, 0.02])
def test_sample_cuts_among_near_equal_logits(vocab, spread):
    """Thousands of logits too near one another for a histogram to tell apart, either side of zero and about 7, with many exact ties."""
    rng = np.random.default_rng(vocab)
    b = 10
    x = (rng.integers(-300, 300, (b, vocab)) * spread / 300).astype(np.float32)
    x[5:] += 7.0
    u = torch.from_numpy(rng.random(b).astype(np.float32))
    k = [1, 255, 256, 257, 1500] * 2
    tok, _, kept, _ = _check(torch.from_numpy(x), u=u, top_k=k)
    assert kept.tolist() == k
    order = np.argsort(-x, axis=1, kind="stable")
    for i in range(b):                                            # all weigh nearly the same: the draw is by place
        rank = np.flatnonzero(np.sort(order[i, :k[i]]) == tok[i])
        assert rank.size == 1 and abs(int(rank[0]) - k[i] * float(u[i])) <= 1 + k[i] * 0.03
    _check(torch.from_numpy(x), u=u, top_p=[0.1, 0.3, 0.5, 0.7, 0.9] * 2)
    _check(torch.from_numpy(x), u=u, top_k=2000, top_p=0.5, min_p=0.5)


@pytest.mark.parametrize("temperature", [1e-30, 1e-6, 1e-3, 50.0, 1e6, 1e30, float("inf")])
def test_sample_temperatures_far_out(temperature):
    rng = np.random.default_rng(9)
    x = torch.from_numpy((rng.standard_normal((9, 40000)) * 3).astype(np.float32))
    u = torch.from_numpy(rng.random(9).astype(np.float32))
    for over in ({}, {"top_k": 700}, {"top_p": 0.6}, {"top_k": 300, "top_p": 0.9}):
        _check(x, u=u, temperature=temperature, **over)
