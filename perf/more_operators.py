"""Measured cases of the operators of a transformer block: attention, the gated projection and the linear layer.

Three operators, each in its plain form (own = False: elementary torch operations in 32 bits,
rounded once at the end) and through the framework's entry points (own = True):

* "attend": softmax attention of q [batch, q, heads, dim] over k, v [batch, kv, kv_heads, dim].
            Every heads / kv_heads consecutive heads share one of k and v. A sequence's own
            lengths say how many of its rows of q and of k and v exist. "causal": query i stands at
            position (length of k) - (length of q) + i and sees the keys up to its own position;
            "window": the last so many of those. A row that sees nothing is zero, its log sum exp
            minus infinity. Backward: dq, dk, dv, the probabilities formed again.
* "gated":  act(x gate^T) * (x up^T), backward to x and both weights.
* "linear": act(x weight^T + bias) + residual, backward to x, weight and bias.

"pass" says which direction a case runs: "forward", or "train" for both.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # One token of a small model over a short cache: launches and latency.
        {"name": "attend_token_small", "op": "attend", "pass": "forward", "batch": 1, "q": 1, "kv": 333, "heads": 8,
         "kv_heads": 8, "dim": 64, "causal": True, "window": 0, "spread": 0.0, "padded_q": False, "dtype": "fp32"},
        # A step of generation for 32 sequences of different lengths, four heads to a key: the cache is read once.
        {"name": "attend_token_cache", "op": "attend", "pass": "forward", "batch": 32, "q": 1, "kv": 8192, "heads": 32,
         "kv_heads": 8, "dim": 128, "causal": True, "window": 0, "spread": 0.5, "padded_q": False, "dtype": "bf16"},
        # A training batch of four sequences of 4096.
        {"name": "attend_train", "op": "attend", "pass": "train", "batch": 4, "q": 4096, "kv": 4096, "heads": 16,
         "kv_heads": 16, "dim": 128, "causal": True, "window": 0, "spread": 0.0, "padded_q": False, "dtype": "bf16"},
        # A padded batch with shared heads and a sliding window; lengths and head size are no power of two.
        {"name": "attend_train_window", "op": "attend", "pass": "train", "batch": 5, "q": 2011, "kv": 2011,
         "heads": 12, "kv_heads": 4, "dim": 80, "causal": True, "window": 512, "spread": 0.6, "padded_q": True,
         "dtype": "bf16"},
        # Cross attention in fp32 to memories of different lengths, one of them empty.
        {"name": "attend_cross_fp32", "op": "attend", "pass": "train", "batch": 3, "q": 777, "kv": 1301, "heads": 6,
         "kv_heads": 2, "dim": 40, "causal": False, "window": 0, "spread": 1.0, "padded_q": False, "dtype": "fp32"},
        # Three tokens of a generation step through both projections: the weights are read once.
        {"name": "gated_token", "op": "gated", "pass": "forward", "tokens": 3, "cols": 2048, "out": 8192,
         "act": "silu", "dtype": "bf16"},
        # A training batch through the gated half of a feed-forward block: the largest case.
        {"name": "gated_train", "op": "gated", "pass": "train", "tokens": 8192, "cols": 2048, "out": 8192,
         "act": "silu", "dtype": "bf16"},
        # Nothing a multiple of anything, fp32.
        {"name": "gated_odd_fp32", "op": "gated", "pass": "train", "tokens": 1201, "cols": 611, "out": 1777,
         "act": "gelu", "dtype": "fp32"},
        # The output projection of one token, added to its residual.
        {"name": "linear_token", "op": "linear", "pass": "forward", "tokens": 1, "cols": 4096, "out": 4096,
         "act": "none", "bias": False, "residual": True, "dtype": "bf16"},
        # The way back from the feed-forward block, added to the residual stream.
        {"name": "linear_train", "op": "linear", "pass": "train", "tokens": 8192, "cols": 8192, "out": 2048,
         "act": "none", "bias": False, "residual": True, "dtype": "bf16"},
        # The first layer of an ungated block, bias and activation in the product.
        {"name": "linear_act_train", "op": "linear", "pass": "train", "tokens": 4096, "cols": 1024, "out": 4096,
         "act": "gelu", "bias": True, "residual": False, "dtype": "bf16"},
        # Nothing a multiple of anything, fp32, with everything.
        {"name": "linear_odd_fp32", "op": "linear", "pass": "train", "tokens": 2003, "cols": 1001, "out": 1501,
         "act": "silu", "bias": True, "residual": True, "dtype": "fp32"},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "gated", "linear"])
    dtype = rng.choice(["fp32", "bf16"])
    way = rng.choice(["forward", "train", "train"])
    if op == "attend":
        group, kv_heads = rng.choice([1, 1, 2, 3, 4, 8]), rng.randint(1, 8)
        heads = group * kv_heads
        dim = rng.choice([64, 128, 8 * rng.randint(1, 16), rng.randint(1, 128)])
        batch = _log_int(rng, 1, 32)
        room = (1 << 29) // (batch * heads)
        if way == "forward" and rng.random() < 0.5:        # generation: few queries over a cache
            q = rng.choice([1, 1, 2, 5, 16])
            kv = _log_int(rng, q, min(65536, room // q, (1 << 29) // (batch * heads * dim)))
        else:
            q = _log_int(rng, 1, min(4096, room))
            kv = q if rng.random() < 0.6 else _log_int(rng, 1, min(4096, room // q))
            kv = min(kv, max(1, room // q))
        if way == "train":     # one key alone has a gradient of nothing but roundings
            kv = max(kv, 2)
        causal = rng.random() < 0.7
        return {"op": op, "pass": way, "batch": batch, "q": q, "kv": kv, "heads": heads, "kv_heads": kv_heads,
                "dim": dim, "causal": causal, "window": _log_int(rng, 2, kv) if causal and rng.random() < 0.3 else 0,
                "spread": rng.choice([0.0, 0.4, 1.0]), "padded_q": q == kv and rng.random() < 0.5, "dtype": dtype}
    # Products of at most a quarter of the largest listed one's (they are three times as slow in fp32).
    cols, out = _log_int(rng, 8, 8192), _log_int(rng, 8, 8192)
    most = (8192 * 2048 * 8192) // 4
    tokens = _log_int(rng, 1, max(2, min(16384, most // (cols * out), (1 << 27) // max(cols, out))))
    case = {"op": op, "pass": way, "tokens": tokens, "cols": cols, "out": out,
            "act": rng.choice(["silu", "gelu", "sigmoid"] + (["relu"] if dtype == "bf16" else []) +
                              (["none"] if op == "linear" else [])), "dtype": dtype}
    if op == "linear":
        case.update(bias=rng.random() < 0.5, residual=rng.random() < 0.5)
    return case


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(gen, shape, scale, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _lengths(case, full):
    """Lengths of a batch's sequences, evenly from the whole down to (1 - spread) of it."""
    n = case["batch"]
    return [int(round(full * (1 - case["spread"] * i / max(1, n - 1)))) for i in range(n)]


def _own_ops():
    from paper_2310_12298_amd import lm
    return lm


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 6271 + 29)
    dt = _dtype(case)
    s = {"case": dict(case)}
    if case["op"] == "attend":
        b, q, kv, h, hk, d = (case[n] for n in ("batch", "q", "kv", "heads", "kv_heads", "dim"))
        if q == kv:            # self attention: the three lie side by side, as one projection leaves them
            rows = _normal(gen, (b, q, h + 2 * hk, d), 1.0, dt)
            s["q"], s["k"], s["v"] = rows[:, :, :h], rows[:, :, h:h + hk], rows[:, :, h + hk:]
        else:
            s["q"] = _normal(gen, (b, q, h, d), 1.0, dt)
            s["k"], s["v"] = (_normal(gen, (b, kv, hk, d), 1.0, dt) for _ in range(2))
        s["kv_lengths"] = s["q_lengths"] = None
        if case["spread"]:
            order = torch.randperm(b, generator=gen, device="cuda")
            s["kv_lengths"] = torch.tensor(_lengths(case, kv), device="cuda")[order]
            if case["padded_q"]:
                s["q_lengths"] = s["kv_lengths"]
        if case["pass"] == "train":
            s["dout"] = _normal(gen, (b, q, h, d), 1e-2, dt)
        return s
    n, d, f = case["tokens"], case["cols"], case["out"]
    s["x"] = _normal(gen, (n, d), 1.0, dt)
    names = ("gate", "up") if case["op"] == "gated" else ("weight",)
    for name in names:
        s[name] = _normal(gen, (f, d), 1.0 / math.sqrt(d), dt)
    if case["op"] == "linear":
        s["bias"] = _normal(gen, (f,), 0.3, dt) if case["bias"] else None
        s["residual"] = _normal(gen, (n, f), 1.0, dt) if case["residual"] else None
    if case["pass"] == "train":
        s["dy"] = _normal(gen, (n, f), 1e-2, dt)
    return s


# ------------------------------------------------------------------ the plain forms
def _seen(case, s):
    """[batch, 1, q, kv]: which keys a query sees."""
    b, q, kv = case["batch"], case["q"], case["kv"]
    dev = "cuda"
    kl = s["kv_lengths"] if s["kv_lengths"] is not None else torch.full((b,), kv, device=dev)
    ql = s["q_lengths"] if s["q_lengths"] is not None else torch.full((b,), q, device=dev)
    i, j = torch.arange(q, device=dev)[None, :, None], torch.arange(kv, device=dev)[None, None, :]
    kl, ql = kl[:, None, None], ql[:, None, None]
    seen = (j < kl) & (i < ql)
    if case["causal"]:
        at = kl - ql + i
        seen = seen & (j <= at)
        if case["window"]:
            seen = seen & (j > at - case["window"])
    return seen[:, None]


def _plain_attend(s):
    c = s["case"]
    b, q, kv, h, hk, d = (c[n] for n in ("batch", "q", "kv", "heads", "kv_heads", "dim"))
    g, dt = h // hk, s["q"].dtype
    scale = 1.0 / math.sqrt(d)
    seen = _seen(c, s)

    def heads(t, spread):      # [batch, heads, rows, dim] in 32 bits, shared heads repeated
        t = t.float().transpose(1, 2)
        return t.repeat_interleave(g, 1) if spread else t.contiguous()
    qf, kf, vf = heads(s["q"], False), heads(s["k"], True), heads(s["v"], True)
    z = torch.matmul(qf, kf.transpose(2, 3).contiguous()) * scale
    z = torch.where(seen, z, torch.full_like(z[:1, :1, :1, :1], -math.inf))
    top = z.max(3, keepdim=True).values
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(z - base)
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, vf)
    out = {"out": o.transpose(1, 2).to(dt), "lse": (base + torch.log(total))[..., 0]}
    if c["pass"] == "train":
        do = heads(s["dout"], False)
        dp = torch.matmul(do, vf.transpose(2, 3).contiguous())
        ds = p * (dp - (do * o).sum(3, keepdim=True)) * scale
        dq = torch.matmul(ds, kf)
        dk = torch.matmul(ds.transpose(2, 3).contiguous(), qf).view(b, hk, g, kv, d).sum(2)
        dv = torch.matmul(p.transpose(2, 3).contiguous(), do).view(b, hk, g, kv, d).sum(2)
        out.update({n: t.transpose(1, 2).to(dt) for n, t in (("dq", dq), ("dk", dk), ("dv", dv))})
    return out


def _plain_act(kind, z):
    """act(z) and its derivative."""
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), (z > 0).float()
    if kind == "gelu":
        phi = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    e = 1 / (1 + torch.exp(-z))
    if kind == "sigmoid":
        return e, e * (1 - e)
    return z * e, e * (1 + z * (1 - e))


def _plain_gated(s):
    dt, act = s["x"].dtype, s["case"]["act"]
    x, wg, wu = s["x"].float(), s["gate"].float(), s["up"].float()
    u = x @ wu.t()
    a, da = _plain_act(act, x @ wg.t())
    out = {"y": (a * u).to(dt)}
    if "dy" in s:
        dy = s["dy"].float()
        dg, du = dy * u * da, dy * a
        out.update(dx=(dg @ wg + du @ wu).to(dt), dgate=(dg.t() @ x).to(dt), dup=(du.t() @ x).to(dt))
    return out


def _plain_linear(s):
    dt, c = s["x"].dtype, s["case"]
    x, w = s["x"].float(), s["weight"].float()
    z = x @ w.t()
    if c["bias"]:
        z = z + s["bias"].float()
    y, da = _plain_act(c["act"], z)
    if c["residual"]:
        y = y + s["residual"].float()
    out = {"y": y.to(dt)}
    if "dy" in s:
        dz = s["dy"].float() * da
        out.update(dx=(dz @ w).to(dt), dweight=(dz.t() @ x).to(dt))
        if c["bias"]:
            out["dbias"] = dz.sum(0).to(dt)
    return out


# ------------------------------------------------------------------ the framework's entry points
def _own_attend(lm, s):
    c = s["case"]
    how = dict(causal=c["causal"], window=c["window"] or None, q_lengths=s["q_lengths"], kv_lengths=s["kv_lengths"])
    o, lse = lm.attention_forward(s["q"], s["k"], s["v"], **how)
    out = {"out": o, "lse": lse}
    if c["pass"] == "train":
        out["dq"], out["dk"], out["dv"] = lm.attention_backward(s["dout"], s["q"], s["k"], s["v"], o, lse, **how)
    return out


def _own_gated(lm, s):
    act = s["case"]["act"]
    out = {"y": lm.gated_linear_forward(s["x"], s["gate"], s["up"], activation=act)}
    if "dy" in s:
        out["dx"], out["dgate"], out["dup"] = lm.gated_linear_backward(s["dy"], s["x"], s["gate"], s["up"],
                                                                       activation=act)
    return out


def _own_linear(lm, s):
    act = None if s["case"]["act"] == "none" else s["case"]["act"]
    out = {"y": lm.linear_forward(s["x"], s["weight"], s["bias"], activation=act, residual=s["residual"])}
    if "dy" in s:
        out["dx"], out["dweight"], db = lm.linear_backward(s["dy"], s["x"], s["weight"], s["bias"], activation=act)
        if s["bias"] is not None:
            out["dbias"] = db
    return out


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"attend": _plain_attend, "gated": _plain_gated, "linear": _plain_linear}[op](s)
    return {"attend": _own_attend, "gated": _own_gated, "linear": _own_linear}[op](_own_ops(), s)


# ------------------------------------------------------------------ 64 bits
def _exact_attend(s):
    c = s["case"]
    b, q, kv, h, hk, d = (c[n] for n in ("batch", "q", "kv", "heads", "kv_heads", "dim"))
    f64 = dict(dtype=torch.float64, device="cuda")
    out = {"out": torch.zeros(b, q, h, d, **f64), "lse": torch.full((b, h, q), -math.inf, **f64)}
    train = c["pass"] == "train"
    if train:
        out.update(dq=torch.zeros(b, q, h, d, **f64), dk=torch.zeros(b, kv, hk, d, **f64),
                   dv=torch.zeros(b, kv, hk, d, **f64))
    lengths = [(q if s["q_lengths"] is None else int(s["q_lengths"][n]),
                kv if s["kv_lengths"] is None else int(s["kv_lengths"][n])) for n in range(b)]
    for n, (nq, nk) in enumerate(lengths):
        first = max(0, nq - nk) if c["causal"] else 0          # rows before it see nothing
        if nk == 0 or first >= nq:
            continue
        rows = slice(first, nq)
        hide = torch.zeros(nq - first, nk, dtype=torch.bool, device="cuda")
        if c["causal"]:
            ones = torch.ones(nq - first, nk, dtype=torch.bool, device="cuda")
            edge = nk - nq + first
            hide = torch.triu(ones, edge + 1)
            if c["window"]:
                hide |= torch.tril(ones, edge - c["window"])
        for m in range(h):
            x, y, w = s["q"][n, rows, m].double(), s["k"][n, :nk, m * hk // h].double(), s["v"][n, :nk, m * hk // h].double()
            z = (x @ y.t() / math.sqrt(d)).masked_fill_(hide, -math.inf)
            out["lse"][n, m, rows] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            out["out"][n, rows, m] = p @ w
            if train:
                g = s["dout"][n, rows, m].double()
                gp = g @ w.t()
                gz = p * gp
                gz -= p * gz.sum(1, keepdim=True)
                gz /= math.sqrt(d)
                out["dq"][n, rows, m] = gz @ y
                out["dk"][n, :nk, m * hk // h] += gz.t() @ x
                out["dv"][n, :nk, m * hk // h] += p.t() @ g
    return out


def _exact_act(kind, z):
    z = z.detach().requires_grad_()
    if kind == "gelu":
        a = z * torch.special.ndtr(z)
    else:
        a = {"none": lambda t: t * 1, "relu": torch.relu, "sigmoid": torch.sigmoid,
             "silu": lambda t: t * torch.sigmoid(t)}[kind](z)
    return a.detach(), torch.autograd.grad(a.sum(), z)[0]


def _exact_dense(s):
    c = s["case"]
    x = s["x"].double()
    if c["op"] == "gated":
        wg, wu = s["gate"].double(), s["up"].double()
        a, da = _exact_act(c["act"], x @ wg.t())
        u = x @ wu.t()
        out = {"y": a * u}
        if "dy" in s:
            dg, du = s["dy"].double() * da * u, s["dy"].double() * a
            out.update(dx=torch.cat([dg, du], 1) @ torch.cat([wg, wu], 0), dgate=(x.t() @ dg).t(), dup=(x.t() @ du).t())
        return out
    w = s["weight"].double()
    z = x @ w.t()
    if s["bias"] is not None:
        z += s["bias"].double()
    y, da = _exact_act(c["act"], z)
    out = {"y": y if s["residual"] is None else y + s["residual"].double()}
    if "dy" in s:
        dz = s["dy"].double() * da
        out.update(dx=dz @ w, dweight=(x.t() @ dz).t())
        if s["bias"] is not None:
            out["dbias"] = dz.sum(0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_attend(s) if case["op"] == "attend" else _exact_dense(s)


def _pairs(case):
    """Pairs of a query and a key that it sees, of one head, over the batch."""
    total = 0
    q, kv = case["q"], case["kv"]
    for nk in _lengths(case, kv):
        nq = nk if case["padded_q"] and case["spread"] else q
        if not case["causal"]:
            total += nq * nk
            continue
        first, last = nk - nq + 1, nk                          # keys up to its own, of the first and the last query
        first = max(first, 1)
        most = case["window"] or last
        if last >= first:
            full = max(0, last - max(first, most) + 1)         # queries that see `most`
            part = min(last, most - 1)
            total += full * most + ((first + part) * (part - first + 1) // 2 if part >= first else 0)
    return total


def work(case):
    """Bytes and operations that a pass cannot do without: each input read once, each output written once."""
    e = 2 if case["dtype"] == "bf16" else 4
    train = case["pass"] == "train"
    if case["op"] == "attend":
        d, h, hk = case["dim"], case["heads"], case["kv_heads"]
        keys = sum(_lengths(case, case["kv"]))
        rows = case["batch"] * case["q"]
        if case["causal"] and case["window"]:
            keys = min(keys, case["batch"] * (case["q"] + case["window"]))
        io = rows * h * d * 2 + keys * hk * d * 2
        if train:                                              # dout read; dq, dk, dv written
            io += rows * h * d * 2 + case["batch"] * case["kv"] * hk * d * 2
        return {"bytes": e * io + 4 * rows * h, "flops": 2.0 * _pairs(case) * h * d * (7 if train else 2)}
    n, d, f = case["tokens"], case["cols"], case["out"]
    w = (2 if case["op"] == "gated" else 1) * f
    io = n * d + w * d + n * f
    if case["op"] == "linear" and case["residual"]:
        io += n * f
    if train:
        io += n * f + n * d + w * d
    return {"bytes": e * io, "flops": 2.0 * n * d * w * (3 if train else 1)}
