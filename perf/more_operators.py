"""Timed and compared cases of the operators of a linear-attention layer around the
packed products: the short causal convolution with its carried inputs, the gated
delta rule over a recurrent state (single tokens and whole prompts), and the gated
norm per head before the output projection: the token mixer of the hybrid decoders
whose linear layers the repository's packed products stand for.

`run` computes each operator either with the library's kernels (`own` true) or in a
plain form of elementary torch operations in 32 bits, rounded once at the end.

Tokens of all sequences are packed: sequence b's rows are starts[b] .. starts[b+1] - 1.
Its state sits in slot slots[b] of a pool; a negative slot marks an unused sequence,
whose rows give zeros. Shapes are generic ones for the widths of the repository's
linear stacks: 12 heads of 64 (d 768), 16 heads of 128 (d 2048), 16 key and 32 value
heads of 128 (d 4096)."""

import math

import torch

own = False

NORM_EPS = 1e-6     # of the unit length of q and k
CHUNK = 64          # tokens that the plain form takes at once


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _conv(name, batch, rows, channels, dtype, taps=4, ragged=False, fresh=False, bias=False):
    return {"name": name, "op": "conv", "batch": batch, "rows": rows, "channels": channels, "dtype": dtype, "taps": taps,
            "ragged": ragged, "fresh": fresh, "bias": bias, "idle": 0, "singles": 0}


def _delta(name, batch, rows, k_heads, heads, head_k, head_v, dtype="bf16", ragged=False, fresh=False, raw=True, singles=0, idle=0):
    return {"name": name, "op": "delta", "batch": batch, "rows": rows, "k_heads": k_heads, "heads": heads, "head_k": head_k,
            "head_v": head_v, "dtype": dtype, "ragged": ragged, "fresh": fresh, "raw": raw, "singles": singles, "idle": idle}


def _norm(name, rows, heads, width, dtype, gate):
    return {"name": name, "op": "norm", "rows": rows, "heads": heads, "width": width, "dtype": dtype, "gate": gate}


def listed():
    return [
        # one decoded token of the 9B-class width: q, k and v channels straight from the product (fp32)
        _conv("conv_token", 1, 1, 8192, "f32"),
        # prompts of different lengths from their beginning, BF16 activations
        _conv("conv_prompts", 6, 3000, 8192, "bf16", ragged=True, fresh=True),
        # one decoded token: 4 MB of state, latency alone
        _delta("delta_token", 1, 1, 16, 32, 128, 128),
        # a serving batch of single tokens: 268 MB of state in and out
        _delta("delta_serving", 64, 1, 16, 32, 128, 128),
        # four sequences taking in 16 prompt tokens each, as many as a packed product takes at once
        _delta("delta_rows", 4, 16, 16, 16, 128, 128),
        # the 131M-class width in fp32, a few hundred tokens each, gates computed by the program itself
        _delta("delta_fp32", 3, 777, 12, 12, 64, 64, dtype="f32", ragged=True, fresh=True, raw=False),
        # prompts of different lengths that start together
        _delta("delta_prompts", 5, 3001, 16, 32, 128, 128, ragged=True, fresh=True),
        # a mixed batch: a prompt's next 2000 tokens beside 23 sequences that decode, one place of the batch unused
        _delta("delta_mixed", 25, 2000, 16, 32, 128, 128, singles=24, idle=1),
        # one long document: the largest
        _delta("delta_document", 1, 32768, 16, 32, 128, 128, fresh=True),
        # the norm before the output projection, one token; the gate is a slice of a product's fp32 output
        _norm("norm_token", 1, 32, 128, "bf16", "f32"),
        # and the tokens of a batch of prompts
        _norm("norm_prompts", 8191, 32, 128, "bf16", "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["conv", "delta", "delta", "delta", "delta", "norm"])
    if op == "norm":
        heads, width = rng.choice([1, 4, 12, 16, 32, 48]), rng.choice([64, 128, 128, 256])
        rows = _log_int(rng, 1, 16000 * 32 * 128 // max(32 * 128, heads * width))
        c = _norm("", rows, heads, width, rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32", "none"]))
    elif op == "conv":
        channels = 8 * _log_int(rng, 16, 1500)
        batch = _log_int(rng, 1, 64)
        rows = rng.choice([1, 1, rng.randint(2, 16), _log_int(rng, 17, 4000)])
        rows = max(1, min(rows, 10000 * 8192 // (batch * channels)))
        c = _conv("", batch, rows, channels, rng.choice(["bf16", "f32"]), rng.choice([2, 3, 4, 4]), rng.random() < 0.5,
                  rng.random() < 0.4, rng.random() < 0.3)
    else:
        head_k, head_v = rng.choice([64, 128, 128]), rng.choice([64, 128, 128, 256])
        k_heads = rng.choice([1, 2, 3, 4, 8, 12, 16])
        heads = k_heads * rng.choice([1, 1, 2, 3, 4])
        batch = _log_int(rng, 1, 64)
        rows = rng.choice([1, 1, rng.randint(2, 16), _log_int(rng, 17, 8000), _log_int(rng, 17, 8000)])
        # no draw reads more state, or computes more, than the largest listed cases
        per = heads * head_k * head_v
        batch = max(1, min(batch, 64 * 32 * 128 * 128 // per))
        rows = max(1, min(rows, 16384 * 32 * 128 * 128 // (batch * per)))
        c = _delta("", batch, rows, k_heads, heads, head_k, head_v, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.6,
                   rng.random() < 0.4, rng.random() < 0.7)
        if batch > 3 and rows > 1 and rng.random() < 0.3:
            c["singles"] = rng.randint(1, batch - 1)
        if batch > 3 and rng.random() < 0.2:
            c["idle"] = 1
    return {k: v for k, v in c.items() if k != "name"}


def _lengths(case):
    """Rows of each sequence; the last `singles` of them have one."""
    b, n = case["batch"], case["rows"]
    many = b - case["singles"]
    lens = [max(1, n - (n // 2) * i // max(1, many) - 7 * i) if case["ragged"] else n for i in range(many)]
    return lens + [1] * case["singles"]


def work(case):
    size = {"f32": 4, "bf16": 2, "none": 0}
    if case["op"] == "norm":
        n = case["rows"] * case["heads"] * case["width"]
        return {"bytes": n * (size[case["dtype"]] + size[case["gate"]] + 2) + 4 * case["width"], "flops": 10 * n}
    lens = _lengths(case)
    used = len(lens) - case["idle"]                     # the idle ones are the last: their rows are written, nothing of them is read
    tokens, read = sum(lens), sum(lens[:used])
    carried = (1 if case["fresh"] else 2) * used        # states read and written
    if case["op"] == "conv":
        c = case["channels"]
        return {"bytes": read * c * size[case["dtype"]] + tokens * c * 2 + carried * c * (case["taps"] - 1) * 4 + c * case["taps"] * 4,
                "flops": read * c * (2 * case["taps"] + 5)}
    h, hk, dk, dv = case["heads"], case["k_heads"], case["head_k"], case["head_v"]
    return {"bytes": read * ((2 * hk * dk + h * dv) * size[case["dtype"]] + 2 * h * 4) + tokens * h * dv * 2 + carried * h * dk * dv * 4,
            "flops": read * h * 7.0 * dk * dv}          # k S, the decay, the update and q S of the recurrence


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case, "op": case["op"]}
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    rand = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")  # noqa: E731
    if case["op"] == "norm":
        n, h, d = case["rows"], case["heads"], case["width"]
        s["x"] = (randn(n, h, d) * torch.exp(randn(1, h, 1))).to(DTYPES[case["dtype"]])       # heads of different strength
        s["weight"] = 1.0 + 0.2 * randn(d)
        s["eps"] = 1e-6
        # the gate is a slice of what one product gives for a token
        s["gate"] = None if case["gate"] == "none" else randn(n, 2 * h * d).to(DTYPES[case["gate"]])[:, h * d:].unflatten(1, (h, d))
        if own:
            s["out"] = torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda")
        return s

    lens = _lengths(case)
    b, tokens = len(lens), sum(lens)
    s["starts"] = torch.tensor([sum(lens[:i]) for i in range(b + 1)], dtype=torch.int32, device="cuda")
    n_slots = b + 3
    slots = torch.randperm(n_slots, generator=gen, device="cuda")[:b].to(torch.int32)
    if case["idle"]:
        slots[b - case["idle"]:] = -1
    s["slots"], s["n_slots"] = slots, n_slots
    s["fresh"] = torch.ones(b, dtype=torch.int32, device="cuda") if case["fresh"] else None
    if own:
        import paper_2607_02893_gb300 as vbq
        s["seq"] = vbq.Sequences(b, max(lens), starts=s["starts"], tokens=tokens, slots=s["slots"], fresh=s["fresh"])
    if case["op"] == "conv":
        c, w = case["channels"], case["taps"]
        s["x"] = randn(tokens, c).to(DTYPES[case["dtype"]])
        s["weight"] = randn(c, w) * w ** -0.5
        s["bias"] = 0.1 * randn(c) if case["bias"] else None
        s["state"] = randn(n_slots, w - 1, c)
        if own:
            s["out"] = torch.empty(tokens, c, dtype=torch.bfloat16, device="cuda")
        return s

    h, hk, dk, dv = (case[k] for k in ("heads", "k_heads", "head_k", "head_v"))
    # q, k and v as the convolution leaves them: one row of channels a token, through silu
    qkv = torch.nn.functional.silu(randn(tokens, 2 * hk * dk + h * dv)).to(DTYPES[case["dtype"]])
    s["q"] = qkv[:, :hk * dk].unflatten(1, (hk, dk))
    s["k"] = qkv[:, hk * dk:2 * hk * dk].unflatten(1, (hk, dk))
    s["v"] = qkv[:, 2 * hk * dk:].unflatten(1, (h, dv))
    gates = randn(tokens, 2 * h)
    if case["raw"]:
        # heads that forget within tens of tokens and heads that keep thousands
        s["a_log"] = torch.log(1.0 + 15.0 * rand(h))
        dt = torch.exp(math.log(0.001) + rand(h) * math.log(100.0))
        s["dt_bias"] = dt + torch.log(-torch.expm1(-dt))
    else:
        s["a_log"] = s["dt_bias"] = None
        gates[:, :h] = -torch.exp(1.5 * gates[:, :h] - 4.0)
        gates[:, h:] = torch.sigmoid(gates[:, h:])
    s["decay"], s["beta"] = gates[:, :h], gates[:, h:]
    s["state"] = 0.3 * randn(n_slots, h, dk, dv)
    s["scale"] = dk ** -0.5
    if own:
        s["out"] = torch.empty(tokens, h, dv, dtype=torch.bfloat16, device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)[s["op"]](s)


def _own_conv(s):
    import paper_2607_02893_gb300 as vbq
    vbq.vbq_causal_conv(s["seq"], s["x"], s["weight"], s["state"], bias=s["bias"], silu=True, out=s["out"])
    return {"out": s["out"], "state": s["state"]}


def _own_delta(s):
    import paper_2607_02893_gb300 as vbq
    vbq.vbq_delta_rule(s["seq"], s["state"], s["q"], s["k"], s["v"], s["decay"], s["beta"], a_log=s["a_log"], dt_bias=s["dt_bias"],
                       scale=s["scale"], normalize=True, out=s["out"])
    return {"out": s["out"], "state": s["state"]}


def _own_norm(s):
    import paper_2607_02893_gb300 as vbq
    return vbq.vbq_gated_norm(s["x"], s["gate"], s["weight"], s["eps"], out=s["out"])


def _places(s):
    """The packed rows as (batch, longest): which row stands there, and whether one does."""
    starts = s["starts"].long()
    lens = (starts[1:] - starts[:-1])
    t = torch.arange(max(_lengths(s["case"])), device="cuda")
    there = t < lens[:, None]
    return torch.where(there, starts[:-1, None] + t, torch.zeros_like(t)), there


def _plain_conv(s):
    c = s["case"]
    w, x, carried = c["taps"], s["x"].float(), s["state"]
    rows, there = _places(s)
    used = s["slots"] >= 0
    slot = torch.where(used, s["slots"], torch.zeros_like(s["slots"])).long()
    before = carried[slot]                                           # batch, taps - 1, channels
    if s["fresh"] is not None:
        before = torch.where(s["fresh"][:, None, None] != 0, torch.zeros_like(before), before)
    line = torch.cat((before, x[rows]), 1)
    n = rows.shape[1]
    y = (line.unfold(1, w, 1) * s["weight"]).sum(-1) if s["bias"] is None else (line.unfold(1, w, 1) * s["weight"]).sum(-1) + s["bias"]
    y = y / (1.0 + torch.exp(-y))
    y = torch.where(used[:, None, None], y, torch.zeros_like(y))
    out = torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda")
    out[rows[there]] = y[:, :n][there].to(torch.bfloat16)
    last = there.sum(1)[:, None] + torch.arange(w - 1, device="cuda")
    carried[slot[used]] = line.gather(1, last[:, :, None].expand(-1, -1, x.shape[1]))[used]
    return {"out": out, "state": carried}


def _unit(x):
    return x * torch.rsqrt((x * x).sum(-1, keepdim=True) + NORM_EPS)


def _log_decay(s):
    """The logarithm of each token's decay, and its beta, in 32 bits."""
    a, b = s["decay"].float(), s["beta"].float()
    if s["a_log"] is None:
        return a, b
    z = a + s["dt_bias"]
    return -torch.exp(s["a_log"]) * (z.clamp(min=0) + torch.log1p(torch.exp(-z.abs()))), 1.0 / (1.0 + torch.exp(-b))


def _plain_delta(s):
    """64 tokens at once. With G_i the sum of the chunk's log decays up to token i and S the state before the chunk, the tokens' corrections solve
    (1 + L) U = beta (V - e^G K S),  L_ij = beta_i e^(G_i - G_j) k_i.k_j below the diagonal; then O = e^G Q S + (e^(G_i - G_j) q_i.k_j, j <= i) U and
    S' = e^(G_last) S + (e^(G_last - G) K)^T U."""
    c = s["case"]
    h, hk, dk, dv = (c[k] for k in ("heads", "k_heads", "head_k", "head_v"))
    rows, there = _places(s)
    b, n = rows.shape
    chunks = -(-n // CHUNK)
    pad = chunks * CHUNK - n
    rows = torch.nn.functional.pad(rows, (0, pad))
    there = torch.nn.functional.pad(there, (0, pad))
    used = s["slots"] >= 0
    slot = torch.where(used, s["slots"], torch.zeros_like(s["slots"])).long()
    live = (there & used[:, None])
    group = h // hk

    def cut(x):                                                      # tokens, heads, d -> batch, heads, chunks, 64, d
        x = torch.where(live[:, :, None, None], x[rows], x.new_zeros(()))
        return x.reshape(b, chunks, CHUNK, *x.shape[2:]).permute(0, 3, 1, 2, 4)

    g, beta = _log_decay(s)
    q = cut(_unit(s["q"].float())).repeat_interleave(group, 1) * s["scale"]
    k = cut(_unit(s["k"].float())).repeat_interleave(group, 1)
    v = cut(s["v"].float())
    g, beta = cut(g[:, :, None])[..., 0], cut(beta[:, :, None])[..., 0]
    upto = g.double().cumsum(-1)
    between = (upto[..., :, None] - upto[..., None, :]).float()
    i = torch.arange(CHUNK, device="cuda")
    below, at_or_below = i[:, None] > i, i[:, None] >= i
    decay = torch.exp(torch.where(at_or_below, between, between.new_full((), -math.inf)))
    low = torch.where(below, beta[..., :, None] * decay * torch.matmul(k, k.transpose(-1, -2)), decay.new_zeros(()))
    score = decay * torch.matmul(q, k.transpose(-1, -2))
    from_start, to_end = torch.exp(upto.float()), torch.exp((upto[..., -1:] - upto).float())
    inverse = torch.eye(CHUNK, device="cuda").expand(low.shape).contiguous()
    for r in range(1, CHUNK):
        inverse[..., r, :] -= torch.matmul(low[..., r:r + 1, :r], inverse[..., :r, :])[..., 0, :]
    own_part = torch.matmul(inverse, beta[..., None] * v)
    state_part = torch.matmul(inverse, (beta * from_start)[..., None] * k)
    q, k = q * from_start[..., None], (k * to_end[..., None]).transpose(-1, -2)
    state = s["state"][slot]
    if s["fresh"] is not None:
        state = torch.where(s["fresh"][:, None, None, None] != 0, torch.zeros_like(state), state)
    o = torch.empty(b, h, chunks, CHUNK, dv, device="cuda")
    for j in range(chunks):
        u = own_part[:, :, j] - torch.matmul(state_part[:, :, j], state)
        o[:, :, j] = torch.matmul(q[:, :, j], state) + torch.matmul(score[:, :, j], u)
        state = from_start[:, :, j, -1, None, None] * state + torch.matmul(k[:, :, j], u)
    out = torch.zeros(s["v"].shape, dtype=torch.bfloat16, device="cuda")
    out[rows[there]] = torch.where(used[:, None, None, None], o.flatten(2, 3).transpose(1, 2), o.new_zeros(()))[there].to(torch.bfloat16)
    s["state"][slot[used]] = state[used]
    return {"out": out, "state": s["state"]}


def _plain_norm(s):
    x = s["x"].float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * s["weight"]
    if s["gate"] is not None:
        z = s["gate"].float()
        y = y * (z / (1.0 + torch.exp(-z)))
    return y.to(torch.bfloat16)


_run_plain = {"conv": _plain_conv, "delta": _plain_delta, "norm": _plain_norm}
_run_own = {"conv": _own_conv, "delta": _own_delta, "norm": _own_norm}


# ---------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_conv(s):
    w = s["case"]["taps"]
    out = torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda")
    state = s["state"].double()
    weight = s["weight"].double()
    ends = s["starts"].tolist()
    for b, slot in enumerate(s["slots"].tolist()):
        if slot < 0:
            continue
        x = s["x"][ends[b]:ends[b + 1]].double()
        past = torch.zeros_like(state[slot]) if s["fresh"] is not None and int(s["fresh"][b]) else state[slot]
        line = torch.cat((past, x), 0)
        y = torch.zeros_like(x)
        for j in range(w):
            y += line[j:j + x.shape[0]] * weight[:, j]
        if s["bias"] is not None:
            y += s["bias"].double()
        out[ends[b]:ends[b + 1]] = y * torch.sigmoid(y)
        state[slot] = line[-(w - 1):]
    return {"out": out, "state": state}


def _exact_delta(s):
    """Token by token: S <- e^g S; u = beta (v - k S); S <- S + k u; o = q S."""
    c = s["case"]
    h, hk = c["heads"], c["k_heads"]
    state_all = s["state"].double()
    lens = _lengths(c)
    slots = s["slots"].tolist()
    # longest first, so that the sequences that go on are a prefix
    order = sorted((b for b in range(len(lens)) if slots[b] >= 0), key=lambda b: -lens[b])
    where = torch.tensor([slots[b] for b in order], device="cuda")
    first = torch.tensor([int(s["starts"][b]) for b in order], device="cuda")
    state = state_all[where]
    if s["fresh"] is not None:
        state = state * (s["fresh"][torch.tensor(order, device="cuda")] == 0).double()[:, None, None, None]
    a, b = s["decay"].double(), s["beta"].double()
    if s["a_log"] is not None:
        z = a + s["dt_bias"].double()
        a, b = -torch.exp(s["a_log"].double()) * torch.logaddexp(z, torch.zeros_like(z)), torch.sigmoid(b)
    keep = torch.exp(a)
    out = torch.zeros(s["v"].shape, dtype=torch.float64, device="cuda")
    # which of the rows each step takes is known ahead
    left = [sum(1 for i in order if lens[i] > t) for t in range(max(lens[i] for i in order))]
    for t, m in enumerate(left):
        at = first[:m] + t
        q, k, v = (s[n][at].double() for n in "qkv")
        q = q / torch.sqrt(q.square().sum(-1, keepdim=True) + NORM_EPS) * s["scale"]
        k = k / torch.sqrt(k.square().sum(-1, keepdim=True) + NORM_EPS)
        q, k = (x.repeat_interleave(h // hk, 1) for x in (q, k))
        now = state[:m]
        now *= keep[at][:, :, None, None]
        u = b[at][:, :, None] * (v - torch.einsum("bhk,bhkv->bhv", k, now))
        now += k[..., None] * u[..., None, :]
        out[at] = torch.einsum("bhk,bhkv->bhv", q, now)
    state_all[where] = state
    return {"out": out, "state": state_all}


def _exact_norm(s):
    x = s["x"].double()
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * s["weight"].double()
    if s["gate"] is not None:
        z = s["gate"].double()
        y = y * z * torch.sigmoid(z)
    return y


def exact(case, seed):
    if case["op"] == "delta":
        steps = max(_lengths(case))
        moved = sum(_lengths(case)) * case["heads"] * case["head_k"] * case["head_v"] * 8.0 * 10
        if steps * 4e-4 + moved / 3e12 > 20:
            return None                                # token by token, this takes too long
    s = prepare(case, seed)
    return {"conv": _exact_conv, "delta": _exact_delta, "norm": _exact_norm}[case["op"]](s)
