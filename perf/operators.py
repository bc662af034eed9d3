"""Timed and compared cases of the operators that a decode step needs around the
packed products: appending to and attending over a key-value cache held in 4 bits,
the residual addition with its norm, and sampling a token from the head's logits.

`run` computes each operator either with the library's kernels (`own` true) or in a
plain form of elementary torch operations in 32 bits, rounded once at the end.

The cache's numbers are defined apart from any layout: a token's key (value) of one
head is cut into groups of 64; a group has an FP16 scale s = absmax / 7 and codes
q = round-half-even(x / s) in -7..7, so it stands for s * q. Shapes are those of the
linear stacks this repository runs: 12 heads of 64 (d 768), 16 heads of 128 over 2
(d 2048), 32 heads of 128 over 8 (d 4096), vocabularies of 32000 and 128256."""

import math

import torch

own = False

PAGE = 64          # tokens in a page of the cache
GROUP = 64         # values that share a scale
UNIT = 2.0 ** 32   # sampling weights are whole multiples of 2^-32 of the largest


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _attend(name, batch, rows, length, heads, kv_heads, head_dim, window=0, ragged=False):
    return {"name": name, "op": "attend", "batch": batch, "rows": rows, "len": length, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "window": window, "ragged": ragged}


def _append(name, batch, rows, length, heads, kv_heads, head_dim, dtype, rotary):
    return {"name": name, "op": "append", "batch": batch, "rows": rows, "len": length, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "rotary": rotary}


def _norm(name, rows, width, dtype, residual):
    return {"name": name, "op": "norm", "rows": rows, "width": width, "dtype": dtype, "residual": residual}


def _sample(name, batch, vocab, dtype, temperature, top_k, top_p, min_p, mixed=False):
    return {"name": name, "op": "sample", "batch": batch, "vocab": vocab, "dtype": dtype, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "mixed": mixed}


def listed():
    return [
        # one decoded token of the 9B-class shape, its Q, K and V straight from the products (fp32), every dimension rotated
        _append("append_token", 1, 1, 4097, 32, 8, 128, "f32", 128),
        # 16 sequences taking in 16 prompt tokens each, BF16 activations, the first half of each head rotated
        _append("append_prompt", 16, 16, 2000, 32, 8, 128, "bf16", 64),
        # the first steps of a short reply of the 131M-class shape: latency alone
        _attend("attend_short", 1, 1, 100, 12, 12, 64),
        # a small batch of chats on the 1B-class shape, every length different
        _attend("attend_chats", 4, 1, 2999, 16, 2, 128, ragged=True),
        # one long document on the 9B-class shape
        _attend("attend_document", 1, 1, 32768, 32, 8, 128),
        # a prompt's 16-token chunks in two sequences, causal within the chunk, keys within a sliding window
        _attend("attend_chunk", 2, 16, 6001, 32, 8, 128, window=4096, ragged=True),
        # a serving batch at long context: the largest, 570 MB of cache
        _attend("attend_serving", 8, 1, 65536, 32, 8, 128),
        # the norm before a product, one token and a full batch of tokens
        _norm("norm_token", 1, 768, "f32", "f32"),
        _norm("norm_batch", 256, 4096, "f32", "bf16"),
        # an ordinary chat setting on the smaller vocabulary
        _sample("sample_topk", 1, 32000, "f32", 0.8, 50, 0.95, 0.0),
        # nucleus sampling of a whole batch from the larger one
        _sample("sample_nucleus", 16, 128256, "f32", 1.0, 0, 0.9, 0.0),
        # rows of one batch with settings of their own, one of them greedy; BF16 logits, with their ties
        _sample("sample_mixed", 5, 128256, "bf16", 1.3, 40, 0.98, 0.02, mixed=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "norm", "sample", "sample"])
    if op == "norm":
        return {k: v for k, v in _norm("", _log_int(rng, 1, 256), _log_int(rng, 64, 16384), rng.choice(["f32", "bf16"]),
                                       rng.choice(["f32", "bf16", "none"])).items() if k != "name"}
    if op == "sample":
        c = _sample("", _log_int(rng, 1, 16), _log_int(rng, 1000, 200000), rng.choice(["f32", "bf16"]),
                    round(rng.uniform(0.3, 1.6), 3), rng.choice([0, 0, 1, 20, 64, 400, 5000]),
                    rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]), rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.2), 4)]),
                    rng.random() < 0.3)
        return {k: v for k, v in c.items() if k != "name"}
    head_dim = rng.choice([64, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 12])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 8])
    if op == "append":
        rotary = rng.choice([0, 32, 64, head_dim])
        c = _append("", _log_int(rng, 1, 16), rng.choice([1, 1, rng.randint(2, 16)]), _log_int(rng, 17, 20000), heads,
                    kv_heads, head_dim, rng.choice(["f32", "bf16"]), rotary)
        return {k: v for k, v in c.items() if k != "name"}
    batch = _log_int(rng, 1, 32)
    rows = rng.choice([1, 1, 1, 2, 5, rng.randint(2, 16)])
    # no draw reads more cache, or computes more, than the largest listed case
    per_token = batch * kv_heads * head_dim
    most = 8 * 65536 * 8 * 128 // per_token
    most = min(most, 131072, 8 * 65536 * 32 * 128 // max(1, batch * rows * heads * head_dim))
    c = _attend("", batch, rows, _log_int(rng, rows, max(rows, most)), heads, kv_heads, head_dim,
                rng.choice([0, 0, 0, _log_int(rng, 16, 8192)]), rng.random() < 0.5)
    return {k: v for k, v in c.items() if k != "name"}


def _lengths(case):
    """Tokens held for each sequence, the new ones among them."""
    b, n = case["batch"], case["len"]
    if not case.get("ragged"):
        return [n] * b
    return [max(case["rows"], n - (n // 2) * i // b - 7 * i) for i in range(b)]


def _keys_read(case):
    """Cached tokens that some row of a sequence attends to, over all sequences."""
    total = 0
    for n in _lengths(case):
        lo = max(0, n - case["rows"] + 1 - case["window"]) if case["window"] else 0
        total += n - lo
    return total


def work(case):
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        size = {"f32": 4, "bf16": 2, "none": 0}
        moved = size[case["dtype"]] + 2 * size[case["residual"]] + 2
        return {"bytes": n * moved + 4 * case["width"], "flops": 5 * n}
    if case["op"] == "sample":
        n = case["batch"] * case["vocab"]
        return {"bytes": n * (4 if case["dtype"] == "f32" else 2), "flops": 8 * n}
    rows, d = case["batch"] * case["rows"], case["head_dim"]
    kv = case["kv_heads"] * (d // 2 + 2 * (d // GROUP)) * 2          # a token's keys and values in the cache
    if case["op"] == "append":
        vals = (case["heads"] + 2 * case["kv_heads"]) * d
        # read the new rows, write q and the cache's form, and read that back as the 32-bit values it stands for
        moved = vals * (4 if case["dtype"] == "f32" else 2) + case["heads"] * d * 2 + kv * 2 + 2 * case["kv_heads"] * d * 4
        return {"bytes": rows * (moved + case["rotary"] * 4), "flops": rows * vals * 8}
    keys = _keys_read(case)
    return {"bytes": keys * kv + 2 * rows * case["heads"] * d * 2,
            "flops": 4.0 * keys * case["rows"] * case["heads"] * d}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _quantise(x):
    """x (..., d) in 32 bits -> FP16 scales (..., d / 64) and codes (..., d), whole numbers in float."""
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    a = g.abs()
    s = (a.amax(-1) / a.new_full((), 7.0)).to(torch.float16)
    # the decision thresholds (j + 1/2) s are exact in 32 bits: no quotient is rounded; a tie goes to the even code
    j = torch.arange(7, device=x.device, dtype=torch.float32)
    edge = s.float()[..., None] * (j + 0.5)
    a, edge = a[..., None], edge[..., None, :]
    up = (a > edge) | ((a == edge) & (j % 2 == 1) & (edge > 0))
    return s, (up.sum(-1) * g.sign()).reshape(x.shape)


def _quantise_bf16(x):
    """The same for BF16 values, whose 32-bit quotients by an FP16 scale are never rounded across a half."""
    g = x.float().reshape(*x.shape[:-1], -1, GROUP)
    s = (g.abs().amax(-1) / g.new_full((), 7.0)).to(torch.float16)
    q = torch.where(s[..., None] > 0, (g / s.float()[..., None]).round(), torch.zeros_like(g))
    return s, q.reshape(x.shape)


def _nibbles(q):
    """Codes -7..7 (..., d) -> two to a byte (..., d / 2), offset by 8."""
    u = (q + 8).to(torch.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4)


def _values(packed, scales):
    """What packed codes and scales stand for, in 32 bits."""
    u = torch.stack((packed & 15, packed >> 4), -1).reshape(*packed.shape[:-1], -1, GROUP)
    v = (u.float() - 8.0) * scales.float()[..., None]
    return v.reshape(*packed.shape[:-1], -1)


def _table(case, gen):
    """A page table over shuffled pages: sequence b's page i."""
    need = [-(-n // PAGE) for n in _lengths(case)]
    per, total = max(need), sum(need)
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(case["batch"], per, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def _positions(case):
    rows = case["rows"]
    return torch.tensor([[n - rows + t for t in range(rows)] for n in _lengths(case)], dtype=torch.int32, device="cuda")


def _history(case, gen):
    """The keys and values of every sequence, in pieces of at most 16384 tokens: (sequence, first token, k, v)."""
    hk, d = case["kv_heads"], case["head_dim"]
    # a few channels of a key are several times larger than the rest
    gain = 1.0 + 3.0 * (torch.rand(hk, d, generator=gen, device="cuda") > 0.95)
    for b, n in enumerate(_lengths(case)):
        for t in range(0, n, 16384):
            m = min(16384, n - t)
            k = torch.randn(m, hk, d, generator=gen, device="cuda") * gain
            v = torch.randn(m, hk, d, generator=gen, device="cuda")
            yield b, t, k.to(torch.bfloat16), v.to(torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case, "op": case["op"]}
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        s["x"] = randn(rows, width).to(DTYPES[case["dtype"]])
        # the residual stream of a deep layer: larger than what a layer adds, some features far larger
        s["residual"] = None if case["residual"] == "none" else \
            (randn(rows, width) * (4.0 + 40.0 * (torch.rand(width, generator=gen, device="cuda") > 0.99))).to(DTYPES[case["residual"]])
        s["weight"] = 1.0 + 0.2 * randn(width)
        s["eps"] = 1e-5
        if own:
            s["out"] = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
            s["residual_out"] = None if s["residual"] is None else torch.empty_like(s["residual"])
        return s
    if case["op"] == "sample":
        b, n = case["batch"], case["vocab"]
        logits = 2.0 * randn(b, n)
        # a head's logits: a wide bulk and a few dozen plausible tokens
        hot = torch.randint(0, n, (b, 64), generator=gen, device="cuda")
        logits.scatter_add_(1, hot, 6.0 * torch.rand(b, 64, generator=gen, device="cuda") + 2.0)
        s["logits"] = logits.to(DTYPES[case["dtype"]])
        row = torch.arange(b, device="cuda")
        full = lambda v, t: torch.full((b,), v, dtype=t, device="cuda")  # noqa: E731
        s["temperature"] = full(case["temperature"], torch.float32)
        s["top_k"] = full(case["top_k"], torch.int32)
        s["top_p"] = full(case["top_p"], torch.float32)
        s["min_p"] = full(case["min_p"], torch.float32)
        if case["mixed"]:
            s["temperature"][row % 5 == 1] = 0.0       # greedy
            s["top_k"][row % 5 == 2] = 0
            s["top_p"][row % 5 == 3] = 1.0
            s["min_p"][row % 5 == 4] = 0.0
        s["u"] = torch.rand(b, generator=gen, device="cuda")
        if own:
            s["tokens"] = torch.empty(b, dtype=torch.int32, device="cuda")
            s["probs"] = torch.empty(b, dtype=torch.float32, device="cuda")
            s["kept"] = torch.empty(b, dtype=torch.int32, device="cuda")
        return s

    b, t, h, hk, d = (case[k] for k in ("batch", "rows", "heads", "kv_heads", "head_dim"))
    s["table"], pages = _table(case, gen)
    s["pos"] = _positions(case)
    if own:
        import paper_2607_02893_gb300 as vbq
        s["cache"] = vbq.KvCache(pages, hk, d)
    else:
        s["k_codes"], s["v_codes"] = (torch.zeros(pages, PAGE, hk, d // 2, dtype=torch.uint8, device="cuda") for _ in "kv")
        s["k_scales"], s["v_scales"] = (torch.zeros(pages, PAGE, hk, d // GROUP, dtype=torch.float16, device="cuda") for _ in "kv")
    if case["op"] == "append":
        s["qkv"] = randn(b, t, (h + 2 * hk) * d).to(DTYPES[case["dtype"]])
        r = case["rotary"]
        if r:
            angle = torch.arange(case["len"], device="cuda", dtype=torch.float64)[:, None] * \
                (10000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r))
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        else:
            s["cos"] = s["sin"] = None
        if own:
            s["q_out"] = torch.empty(b, t, h, d, dtype=torch.bfloat16, device="cuda")
            s["k_out"], s["v_out"] = (torch.empty(b, t, hk, d, device="cuda") for _ in "kv")
        return s
    for i, first, k, v in _history(case, gen):
        n = k.shape[0]
        if own:
            pos = torch.arange(first, first + n, dtype=torch.int32, device="cuda")[None]
            vbq.vbq_kv_append(s["cache"], s["table"][i:i + 1], pos, k[None], v[None])
            continue
        at = torch.arange(first, first + n, device="cuda")
        page, slot = s["table"][i, at // PAGE].long(), at % PAGE
        for name, x in (("k", k), ("v", v)):
            scale, q = _quantise_bf16(x)
            s[name + "_codes"][page, slot] = _nibbles(q)
            s[name + "_scales"][page, slot] = scale
    s["q"] = (randn(b, t, h, d) * 1.5).to(torch.bfloat16)
    s["scale"] = d ** -0.5
    if own:
        s["out"] = torch.empty_like(s["q"])
        s["workspace"] = vbq.vbq_kv_workspace(s["cache"], b, t, h)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)[s["op"]](s)


def _rotate(x, c, sn):
    """Rotates the pairs (i, i + r / 2) of the first r dimensions of x (b, t, heads, d); c, sn (b, t, 1, r / 2)."""
    half = c.shape[-1]
    a, b = x[..., :half], x[..., half:2 * half]
    return torch.cat((a * c - b * sn, b * c + a * sn, x[..., 2 * half:]), -1)


def _plain_append(s):
    c = s["case"]
    b, t, h, hk, d = (c[k] for k in ("batch", "rows", "heads", "kv_heads", "head_dim"))
    x = s["qkv"].float().reshape(b, t, h + 2 * hk, d)
    q, k, v = x[:, :, :h], x[:, :, h:h + hk], x[:, :, h + hk:]
    at = s["pos"].long()
    if s["cos"] is not None:
        cos, sin = s["cos"][at][:, :, None], s["sin"][at][:, :, None]
        q, k = _rotate(q, cos, sin), _rotate(k, cos, sin)
    page, slot = s["table"].gather(1, at // PAGE).long(), at % PAGE
    ks, kq = _quantise(k)
    vs, vq = _quantise(v)
    kn, vn = _nibbles(kq), _nibbles(vq)
    s["k_codes"][page, slot], s["v_codes"][page, slot] = kn, vn
    s["k_scales"][page, slot], s["v_scales"][page, slot] = ks, vs
    return {"q": q.to(torch.bfloat16), "k": _values(s["k_codes"][page, slot], s["k_scales"][page, slot]),
            "v": _values(s["v_codes"][page, slot], s["v_scales"][page, slot])}


def _own_append(s):
    import paper_2607_02893_gb300 as vbq
    c = s["case"]
    b, t, h, hk, d = (c[k] for k in ("batch", "rows", "heads", "kv_heads", "head_dim"))
    x = s["qkv"].view(b, t, h + 2 * hk, d)
    vbq.vbq_kv_append(s["cache"], s["table"], s["pos"], x[:, :, h:h + hk], x[:, :, h + hk:], q=x[:, :, :h],
                      q_out=s["q_out"], cos=s["cos"], sin=s["sin"])
    vbq.vbq_kv_read(s["cache"], s["table"], s["pos"], k_out=s["k_out"], v_out=s["v_out"])
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _plain_attend(s):
    c = s["case"]
    b, t, h, hk, d = (c[k] for k in ("batch", "rows", "heads", "kv_heads", "head_dim"))
    table = s["table"].long()
    n = table.shape[1] * PAGE
    k = _values(s["k_codes"][table], s["k_scales"][table]).reshape(b, n, hk, d).permute(0, 2, 3, 1)
    v = _values(s["v_codes"][table], s["v_scales"][table]).reshape(b, n, hk, d).permute(0, 2, 1, 3)
    q = s["q"].float().reshape(b, t, hk, h // hk, d).permute(0, 2, 1, 3, 4).reshape(b, hk, -1, d)
    score = torch.matmul(q, k) * s["scale"]                          # b, hk, t * group, n
    pos = s["pos"].repeat_interleave(h // hk, 1)[:, None, :, None]
    at = torch.arange(n, device="cuda", dtype=torch.int32)
    seen = at <= pos
    if c["window"]:
        seen = seen & (at > pos - c["window"])
    score = torch.where(seen, score, score.new_full((), -math.inf))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return out.reshape(b, hk, t, h // hk, d).permute(0, 2, 1, 3, 4).reshape(b, t, h, d).to(torch.bfloat16)


def _own_attend(s):
    import paper_2607_02893_gb300 as vbq
    return vbq.vbq_kv_attend(s["cache"], s["table"], s["pos"], s["q"], scale=s["scale"], window=s["case"]["window"],
                             out=s["out"], workspace=s["workspace"])


def _plain_norm(s):
    x = s["x"].float()
    if s["residual"] is not None:
        new = (s["residual"].float() + x).to(s["residual"].dtype)
        x = new.float()
    else:
        new = None
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * s["weight"]
    return {"out": y.to(torch.bfloat16), "residual": new}


def _own_norm(s):
    import paper_2607_02893_gb300 as vbq
    vbq.vbq_residual_norm(s["x"], s["residual"], s["weight"], s["eps"], out=s["out"], residual_out=s["residual_out"])
    return {"out": s["out"], "residual": s["residual_out"]}


def _plain_sample(s):
    x = s["logits"].float()
    b, n = x.shape
    greedy = s["temperature"] <= 0
    t = torch.where(greedy, torch.ones_like(s["temperature"]), s["temperature"])[:, None]
    z, order = torch.sort(x, dim=-1, descending=True, stable=True)   # ties: the lowest index first
    e = torch.exp((z - z[:, :1]) / t)
    w = torch.round(e * UNIT).to(torch.int64)                        # whole numbers: sums do not depend on order
    rank = torch.arange(n, device="cuda")
    k = torch.where(s["top_k"] > 0, s["top_k"], torch.full_like(s["top_k"], n))
    k = torch.where(greedy, torch.ones_like(k), k)[:, None]
    keep = rank < k
    w = torch.where(keep, w, torch.zeros_like(w))
    upto = w.cumsum(-1)
    enough = s["top_p"].double()[:, None] * upto[:, -1:].double()
    # the shortest prefix whose mass reaches top_p of what top_k left
    keep = keep & ((s["top_p"][:, None] >= 1) | (rank == 0) | ((upto - w).double() < enough))
    keep = keep & (e >= s["min_p"][:, None])
    w = torch.where(keep, w, torch.zeros_like(w))
    by_index = torch.zeros_like(w).scatter_(1, order, w)             # the draw goes through the tokens in index order
    upto = by_index.cumsum(-1)
    total = upto[:, -1:]
    token = (upto.double() <= s["u"].double()[:, None] * total.double()).sum(-1)
    chance = torch.zeros_like(e).scatter_(1, order, e).gather(1, token[:, None])[:, 0] / (total[:, 0].double() / UNIT).float()
    return {"token": token.to(torch.int32), "prob": chance, "kept": keep.sum(-1).to(torch.int32)}


def _own_sample(s):
    import paper_2607_02893_gb300 as vbq
    vbq.vbq_sample(s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"], tokens=s["tokens"],
                   probs=s["probs"], kept=s["kept"])
    return {"token": s["tokens"], "prob": s["probs"], "kept": s["kept"]}


_run_plain = {"append": _plain_append, "attend": _plain_attend, "norm": _plain_norm, "sample": _plain_sample}
_run_own = {"append": _own_append, "attend": _own_attend, "norm": _own_norm, "sample": _own_sample}


# ---------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_quantised(x):
    """What x (..., d), in 64 bits, is held as."""
    out = torch.empty_like(x)
    for g in range(0, x.shape[-1], GROUP):
        y = x[..., g:g + GROUP]
        s = (y.abs().max(-1, keepdim=True).values / 7).to(torch.float16).double()
        out[..., g:g + GROUP] = torch.where(s > 0, s * torch.round(y / s).clamp(-7, 7), torch.zeros_like(y))
    return out


def _exact_append(s):
    c = s["case"]
    h, hk, d, r = c["heads"], c["kv_heads"], c["head_dim"], c["rotary"]
    x = s["qkv"].double().reshape(c["batch"], c["rows"], h + 2 * hk, d).clone()
    if r:
        at = s["pos"].long()
        c64, s64 = s["cos"].double()[at][:, :, None], s["sin"].double()[at][:, :, None]
        turned = x[:, :, :h + hk]
        first, second = turned[..., :r // 2].clone(), turned[..., r // 2:r].clone()
        turned[..., :r // 2] = first * c64 - second * s64
        turned[..., r // 2:r] = second * c64 + first * s64
    return {"q": x[:, :, :h].contiguous(), "k": _exact_quantised(x[:, :, h:h + hk].contiguous()),
            "v": _exact_quantised(x[:, :, h + hk:].contiguous())}


def _exact_attend(s):
    c = s["case"]
    t, h, hk, d = (c[k] for k in ("rows", "heads", "kv_heads", "head_dim"))
    group = h // hk
    out = torch.zeros(c["batch"], t, h, d, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(c)):
        pages = s["table"][b, :-(-n // PAGE)].long()
        for j in range(hk):
            kv = []
            for name in "kv":
                byte = s[name + "_codes"][pages, :, j].reshape(-1, d // 2)[:n].long()
                code = torch.empty(n, d, dtype=torch.float64, device="cuda")
                code[:, 0::2], code[:, 1::2] = (byte % 16 - 8).double(), (byte // 16 - 8).double()
                kv.append(code * s[name + "_scales"][pages, :, j].reshape(-1, d // GROUP)[:n].double().repeat_interleave(GROUP, 1))
            for i in range(t):
                p = int(s["pos"][b, i])
                lo = max(0, p + 1 - c["window"]) if c["window"] else 0
                if p < lo:
                    continue
                q = s["q"][b, i, j * group:(j + 1) * group].double()
                a = torch.softmax(q @ kv[0][lo:p + 1].T * s["scale"], -1)
                out[b, i, j * group:(j + 1) * group] = a @ kv[1][lo:p + 1]
    return out


def _exact_norm(s):
    x = s["x"].double()
    new = None
    if s["residual"] is not None:
        # the norm is defined on the residual stream as it is stored: the sum of two 32-bit values, rounded to its type
        new = (s["residual"].double() + x).float().to(s["residual"].dtype).double()
        x = new
    return {"out": x / torch.sqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * s["weight"].double(), "residual": new}


def _exact_sample(s):
    x = s["logits"].double()
    prob, n = [], x.shape[1]
    for b in range(x.shape[0]):
        top, t = x[b].max(), float(s["temperature"][b])
        if t <= 0:
            prob.append(1.0)
            continue
        e = torch.exp((x[b] - top) / t)
        order = torch.argsort(x[b], descending=True, stable=True)
        k = int(s["top_k"][b])
        order = order[:k] if k > 0 else order
        p = float(s["top_p"][b])
        if p < 1:
            mass = e[order].cumsum(0)
            order = order[:max(1, int((mass < p * mass[-1]).sum()) + 1)]
        order = order[e[order] >= float(s["min_p"][b])]
        order = order.sort().values
        mass = e[order].cumsum(0)
        at = min(int((mass <= float(s["u"][b]) * mass[-1]).sum()), order.numel() - 1)
        prob.append(float(e[order[at]] / mass[-1]))
    return {"token": None, "prob": torch.tensor(prob, dtype=torch.float64), "kept": None}


def exact(case, seed):
    if case["op"] == "attend" and case["batch"] * case["rows"] * case["kv_heads"] > 6000:
        return None                                    # the loops below would take too long
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "norm": _exact_norm, "sample": _exact_sample}[case["op"]](s)
