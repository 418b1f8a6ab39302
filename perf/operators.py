"""Measured cases of the operators of a language model's training step that stand beside the Jorge step.

Four operators, each in its plain form (own = False: elementary torch operations in
32 bits, rounded once at the end) and through the framework's entry points (own = True):

* "norm":  layer norm, forward, and backward with the reduction of the gain's and the
           bias's gradient over the rows;
* "embed": embedding lookup with scaling, and its gradient with respect to the table;
* "loss":  softmax cross entropy of hidden @ weight.T over a vocabulary, forward, and
           backward to both operands;
* "adamw": one AdamW step over many tensors, with moments in 32 bits or in 8 (blocks of
           256 with a power-of-two scale, rounded by random bits made from a seed, the
           step and the element's place), with or without clipping by the global norm.

"pass" says which direction a case runs: "forward", or "train" for both.

The 8-bit moments. A block of 256 consecutive elements of a tensor has one scale byte
k, standing for 2^(k - 127), k in 1 .. 253: the least k with max|x| <= 31/16 2^(k - 127).
An element's code is a small float y with x = y 2^(k - 127):
  first moment:  1 sign bit, 3 exponent bits E, 4 mantissa bits M:
                 y = (1 + M/16) 2^(E - 7) for E > 0, (M/16) 2^-6 for E = 0;
  second moment: 4 exponent bits E, 4 mantissa bits M:
                 y = (1 + M/16) 2^(E - 15) for E > 0, (M/16) 2^-14 for E = 0.
x / 2^(k - 127) is rounded to one of its two neighbours: up where the part between them,
in units of 2^-16 and cut off, plus the element's 16 random bits reaches 2^16. A second
moment above zero keeps at least the smallest code, so that no step divides by eps alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

F32_EPS = 1e-5             # layer norm's epsilon
IGNORE = -100              # a target that stands for no target
ADAM = dict(lr=3e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
BLOCK = 256                # elements of an 8-bit moment that share a scale
MASK32 = 0xFFFFFFFF


def listed():
    return [
        # Normalising a handful of rows, as in generation or a small batch: latency.
        {"name": "norm_few_rows", "op": "norm", "pass": "forward", "rows": 7, "cols": 1024, "dtype": "fp32"},
        # Every token of a training batch through one layer norm of a 4096-wide model, both directions.
        {"name": "norm_train", "op": "norm", "pass": "train", "rows": 16384, "cols": 4096, "dtype": "bf16"},
        # A width and a row count that are no multiple of anything.
        {"name": "norm_odd", "op": "norm", "pass": "train", "rows": 5003, "cols": 1999, "dtype": "fp32"},
        # The embedding of a training batch: 16384 tokens of a 50000-word vocabulary, Zipf-distributed.
        {"name": "embed_train", "op": "embed", "pass": "train", "tokens": 16384, "vocab": 50000, "cols": 2048,
         "dtype": "bf16", "pad": 0.0},
        # A batch that is half padding: one row of the table takes half of all tokens.
        {"name": "embed_padded", "op": "embed", "pass": "train", "tokens": 65536, "vocab": 8192, "cols": 512,
         "dtype": "fp32", "pad": 0.5},
        # The loss of a few tokens of a small model: launches and latency.
        {"name": "loss_small", "op": "loss", "pass": "train", "tokens": 64, "cols": 512, "vocab": 8192,
         "dtype": "fp32", "smoothing": 0.0, "ignored": 0.0},
        # Evaluation: the loss alone.
        {"name": "loss_eval", "op": "loss", "pass": "forward", "tokens": 4096, "cols": 2048, "vocab": 32768,
         "dtype": "bf16", "smoothing": 0.0, "ignored": 0.0},
        # The loss of a training batch over an odd vocabulary, a tenth of the targets masked: the largest case.
        {"name": "loss_train", "op": "loss", "pass": "train", "tokens": 8192, "cols": 2048, "vocab": 50001,
         "dtype": "bf16", "smoothing": 0.0, "ignored": 0.1},
        # The same in fp32 with label smoothing, nothing a multiple of anything.
        {"name": "loss_odd_fp32", "op": "loss", "pass": "train", "tokens": 2001, "cols": 1001, "vocab": 30011,
         "dtype": "fp32", "smoothing": 0.1, "ignored": 0.05},
        # The gains and biases of a small model: many tiny tensors, latency.
        {"name": "adamw_vectors", "op": "adamw", "net": "vectors", "layers": 50, "width": 512, "bits": 32,
         "dtype": "fp32", "clip": False},
        # Every weight matrix of ResNet-50, clipped by the global norm.
        {"name": "adamw_resnet50", "op": "adamw", "net": "resnet50", "layers": 54, "width": 0, "bits": 32,
         "dtype": "fp32", "clip": True},
        # The framework's set of large dense layers (168 M weights) with 8-bit moments.
        {"name": "adamw_dense_8bit", "op": "adamw", "net": "dense", "layers": 8, "width": 4096, "bits": 8,
         "dtype": "fp32", "clip": False},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "embed", "loss", "adamw"])
    dtype = rng.choice(["fp32", "bf16"])
    way = rng.choice(["forward", "train", "train"])
    if op == "norm":
        cols = _log_int(rng, 1, 16384)
        return {"op": op, "pass": way, "rows": _log_int(rng, 1, max(2, min(65536, (1 << 26) // cols))), "cols": cols,
                "dtype": dtype}
    if op == "embed":
        cols = _log_int(rng, 8, 8192)
        vocab = _log_int(rng, 2, min(200000, (1 << 27) // cols))
        return {"op": op, "pass": way, "tokens": _log_int(rng, 1, max(2, min(131072, (1 << 26) // cols))),
                "vocab": vocab, "cols": cols, "dtype": dtype, "pad": rng.choice([0.0, 0.0, 0.3, 0.9])}
    if op == "loss":
        cols = _log_int(rng, 16, 4096)
        vocab = _log_int(rng, 10, 100000)
        # fp32 products cost six times as much: a drawn case stays below the largest listed one.
        most = (8192 * 2048 * 50001) // (6 if dtype == "fp32" else 1)
        return {"op": op, "pass": way, "tokens": _log_int(rng, 1, max(2, min(16384, most // (cols * vocab)))),
                "cols": cols, "vocab": vocab, "dtype": dtype, "smoothing": rng.choice([0.0, 0.0, 0.1]),
                "ignored": rng.choice([0.0, 0.1, 0.6])}
    return {"op": op, "net": "ragged", "layers": rng.randint(1, 80), "width": _log_int(rng, 16, 2048),
            "seed": rng.randint(0, 99), "bits": rng.choice([8, 32]), "dtype": dtype, "clip": rng.random() < 0.5}


def _numels(case):
    """Elements of each tensor of an "adamw" case."""
    if case["net"] == "vectors":
        return [case["width"]] * case["layers"]
    if case["net"] == "dense":
        w = case["width"]
        return [w * w] * case["layers"] + [w * w // 4] * case["layers"]
    if case["net"] == "ragged":
        import random
        r = random.Random(case["seed"])
        return [_log_int(r, 1, case["width"] * case["width"]) for _ in range(case["layers"])]
    numels, width = [64 * 147], 64                             # ResNet-50: stem, bottlenecks, classifier
    for w, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
        for b in range(blocks):
            numels += [w * width, 9 * w * w, 4 * w * w] + ([4 * w * width] if b == 0 else [])
            width = 4 * w
    return numels + [1000 * 2048]


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(gen, shape, scale, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _zipf(gen, count, vocab, pad):
    """Tokens whose frequency falls as one over their rank, ranks in a random order of rows; `pad` of them are row 0."""
    u = torch.rand(count, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    tok = torch.randperm(vocab, generator=gen, device="cuda")[rank]
    if pad:
        tok[torch.rand(count, generator=gen, device="cuda") < pad] = 0
    return tok


def _own_ops():
    from paper_2310_12298_amd import lm
    return lm


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    dt = _dtype(case)
    s = {"case": dict(case)}
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        # A residual stream: every row with its own scale and offset.
        x = _normal(gen, (rows, cols), 1.0)
        x *= torch.rand((rows, 1), generator=gen, device="cuda") * 2 + 0.2
        x += _normal(gen, (rows, 1), 0.3)
        s["x"] = x.to(dt)
        s["weight"] = 1.0 + _normal(gen, (cols,), 0.1)
        s["bias"] = _normal(gen, (cols,), 0.1)
        if case["pass"] == "train":
            s["dy"] = _normal(gen, (rows, cols), 1e-2, dt)
        return s
    if case["op"] == "embed":
        s["tokens"] = _zipf(gen, case["tokens"], case["vocab"], case["pad"])
        s["table"] = _normal(gen, (case["vocab"], case["cols"]), 0.02, dt)
        s["scale"] = math.sqrt(case["cols"])
        if case["pass"] == "train":
            s["dout"] = _normal(gen, (case["tokens"], case["cols"]), 1e-3, dt)
        return s
    if case["op"] == "loss":
        n, d, v = case["tokens"], case["cols"], case["vocab"]
        s["hidden"] = _normal(gen, (n, d), 1.0, dt)
        # Logits of a model part-way through training: a spread of about two.
        s["weight"] = _normal(gen, (v, d), 2.0 / math.sqrt(d), dt)
        t = _zipf(gen, n, v, 0.0)
        if case["ignored"]:
            t[torch.rand(n, generator=gen, device="cuda") < case["ignored"]] = IGNORE
        s["targets"] = t
        s["grad"] = torch.ones((), device="cuda")
        return s
    numels = _numels(case)
    # One flat buffer each for weights, gradients and moments; a tensor starts a block of 256 elements, and what
    # lies between two tensors is zero and stays so.
    first = [0]
    for n in numels:
        first.append(first[-1] + -(-n // BLOCK) * BLOCK)
    total = first[-1]
    used = torch.zeros(total, dtype=torch.float32, device="cuda")
    size = torch.zeros(total, dtype=torch.float32, device="cuda")
    for i, (f, n) in enumerate(zip(first, numels)):
        used[f: f + n] = 1.0
        size[f: f + n] = 1 + i % 5             # layers whose gradients differ in size
    s["p"] = (_normal(gen, (total,), 0.05) * used).to(dt)
    s["g"] = (_normal(gen, (total,), 1e-3) * size).to(dt)
    m = _normal(gen, (total,), 3e-4) * size
    v = _normal(gen, (total,), 1e-3).mul_(size).square_()
    s["step"] = 101
    s["seed"] = seed & 0xFFFF
    if case["bits"] == 8:
        u = torch.randint(0, 1 << 16, (2, total), generator=gen, device="cuda", dtype=torch.int32)
        s["m"], s["m_scale"] = _encode(m, u[0], True)
        s["v"], s["v_scale"] = _encode(v, u[1], False)
        moments = {"exp_avg": s["m"], "exp_avg_sq": s["v"], "exp_avg_scale": s["m_scale"],
                   "exp_avg_sq_scale": s["v_scale"]}
    else:
        s["m"], s["v"] = m, v
        moments = {"exp_avg": s["m"], "exp_avg_sq": s["v"]}
    s["max_norm"] = 1.0 if case["clip"] else 0.0
    if own:   # the handle that a program keeps over its steps: its tensors, and the moments that a checkpoint gave
        cut = lambda x: [x[f: f + n] for f, n in zip(first, numels)]  # noqa: E731
        s["grads"] = cut(s["g"])
        s["opt"] = _own_ops().AdamW(cut(s["p"]), bits=case["bits"], seed=s["seed"], moments=moments)
    return s


# ------------------------------------------------------------------ the plain forms
def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + F32_EPS)
    xhat = c * rstd
    out = {"y": (xhat * s["weight"] + s["bias"]).to(s["x"].dtype)}
    if "dy" in s:
        dy = s["dy"].float()
        g = dy * s["weight"]
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        out.update(dx=dx.to(s["x"].dtype), dweight=(dy * xhat).sum(0), dbias=dy.sum(0))
    return out


def _plain_embed(s):
    out = {"out": (s["table"][s["tokens"]].float() * s["scale"]).to(s["table"].dtype)}
    if "dout" in s:
        d = torch.zeros(s["table"].shape, dtype=torch.float32, device="cuda")
        d.index_add_(0, s["tokens"], s["dout"].float())
        out["dtable"] = (d * s["scale"]).to(s["table"].dtype)
    return out


def _plain_loss(s):
    c = s["case"]
    h, w, t = s["hidden"].float(), s["weight"].float(), s["targets"]
    eps, vocab = c["smoothing"], c["vocab"]
    z = h @ w.t()
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    live = (t >= 0) & (t < vocab) & (t != IGNORE)
    at = torch.where(live, t, torch.zeros_like(t))
    zt = z.gather(1, at[:, None])[:, 0]
    loss = lse - (1 - eps) * zt - (eps * z.mean(1) if eps else 0.0)
    loss = torch.where(live, loss, torch.zeros_like(loss))
    count = live.sum().clamp(min=1)
    out = {"loss": loss.sum() / count, "rows": loss, "lse": lse}
    if c["pass"] == "train":
        dz = (e / total) - eps / vocab
        dz.scatter_add_(1, at[:, None], torch.full_like(dz[:, :1], eps - 1.0))
        dz *= (live * (s["grad"] / count))[:, None]
        out.update(dhidden=(dz @ w).to(s["hidden"].dtype), dweight=(dz.t() @ h).to(s["weight"].dtype))
    return out


def _random32(index, seed, step):
    """32 random bits for each element: a counter's hash (additions and products modulo 2^32, shifted onto itself)."""
    h = (index & MASK32) * 0x9E3779B1 + (index >> 32) * 0x632BE5AB + seed * 0x85157AF5 + step * 0x2C9277B5
    h = h & MASK32
    h = ((h ^ (h >> 16)) * 0x7C2E1B35) & MASK32
    h = ((h ^ (h >> 15)) * 0x46D8C6A9) & MASK32
    return h ^ (h >> 16)


def _pow2(e):
    """2^e in 32 bits for whole e in -126 .. 127, from its bits."""
    return ((e + 127) << 23).int().view(torch.float32)


def _decode(code, scale, signed):
    """The values that codes and scales of blocks stand for, in 32 bits (exact)."""
    code = code.int()
    mag = (code & 0x7F) if signed else code
    e, man = mag >> 4, (mag & 15).float()
    bias = 7 if signed else 15
    y = torch.where(e > 0, 16 + man, man) * _pow2(e.clamp(min=1) - bias - 4)
    y = (y.view(-1, BLOCK) * _pow2(scale.int() - 127)[:, None]).view(-1)
    return torch.where(code >= 128, -y, y) if signed else y


def _encode(x, bits16, signed):
    """Codes and block scales of 32-bit values, rounded by 16 random bits each."""
    size = x.abs()
    top = size.view(-1, BLOCK).amax(1)
    man, e = torch.frexp(top)                                  # top = man 2^e, man in [1/2, 1)
    k = torch.where(top > 0, (e + 126 + (man > 31 / 32).int()).clamp(1, 253), torch.ones_like(e))
    y = (size.view(-1, BLOCK) * _pow2(127 - k)[:, None]).view(-1)
    bias, least = (7, -6) if signed else (15, -14)
    e = torch.where(y > 0, torch.frexp(y)[1] - 1, least).clamp(min=least)
    fixed = torch.floor(y * _pow2(20 - e)).int()               # 4 mantissa bits and 16 below them
    q = (fixed + bits16.int()) >> 16                           # 16 .. 32 of a normal number, 0 .. 16 below
    code = ((e + bias - 1) << 4) + q                           # a carry moves into the exponent by itself
    if not signed:
        code = torch.where((x > 0) & (code == 0), torch.ones_like(code), code)
    code = code.clamp(max=127 if signed else 255)
    code = torch.where(x < 0, code + 128, code) if signed else code
    return code.to(torch.uint8), k.to(torch.uint8)


def _plain_adamw(s):
    small, t = s["case"]["bits"] == 8, s["step"]
    s["step"] = t + 1
    p, g = s["p"].float(), s["g"].float()
    norm = None
    if s["max_norm"]:
        norm = torch.sqrt((g * g).sum())
        g = g * torch.clamp(s["max_norm"] / norm, max=1.0)
    m = _decode(s["m"], s["m_scale"], True) if small else s["m"]
    v = _decode(s["v"], s["v_scale"], False) if small else s["v"]
    m = m + (g - m) * (1 - ADAM["beta1"])
    v = v + (g * g - v) * (1 - ADAM["beta2"])
    a = ADAM["lr"] / (1 - ADAM["beta1"] ** t)
    r = 1 / math.sqrt(1 - ADAM["beta2"] ** t)
    p = p - (p * (ADAM["lr"] * ADAM["weight_decay"]) + (m * a) / (torch.sqrt(v) * r + ADAM["eps"]))
    s["p"].copy_(p)
    out = {"params": s["p"]}
    if small:
        u = _random32(torch.arange(m.numel(), device="cuda"), s["seed"], t)
        s["m"][:], s["m_scale"][:] = _encode(m, u & 0xFFFF, True)
        s["v"][:], s["v_scale"][:] = _encode(v, u >> 16, False)
        # Five significant bits: a bfloat16 holds such a value exactly.
        out["m"] = _decode(s["m"], s["m_scale"], True).bfloat16()
        out["v"] = _decode(s["v"], s["v_scale"], False).bfloat16()
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out["m"], out["v"] = s["m"], s["v"]
    if norm is not None:
        out["norm"] = norm
    return out


# ------------------------------------------------------------------ the framework's entry points
def _own_adamw(s):
    opt = s["opt"]
    opt.t = s["step"] - 1
    s["step"] += 1
    opt.step(s["grads"], max_norm=s["max_norm"], **ADAM)
    out = {"params": s["p"]}
    if s["case"]["bits"] == 8:
        out["m"], out["v"] = opt.moment_values(torch.bfloat16)
    else:
        out["m"], out["v"] = s["m"], s["v"]
    if s["max_norm"]:
        out["norm"] = opt.norm
    return out


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"norm": _plain_norm, "embed": _plain_embed, "loss": _plain_loss, "adamw": _plain_adamw}[op](s)
    lm = _own_ops()
    train = s["case"].get("pass") == "train"
    if op == "norm":
        y, mean, rstd = lm.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=F32_EPS)
        out = {"y": y}
        if train:
            dx, dw, db = lm.layer_norm_backward(s["dy"], s["x"], mean, rstd, s["weight"])
            out.update(dx=dx, dweight=dw, dbias=db)
        return out
    if op == "embed":
        out = {"out": lm.embedding_forward(s["tokens"], s["table"], scale=s["scale"])}
        if train:
            out["dtable"] = lm.embedding_backward(s["dout"], s["tokens"], s["case"]["vocab"], scale=s["scale"])
        return out
    if op == "loss":
        how = dict(ignore_index=IGNORE, label_smoothing=s["case"]["smoothing"])
        rows, lse, total = lm.cross_entropy_forward(s["hidden"], s["weight"], s["targets"], **how)
        out = {"loss": total[2], "rows": rows, "lse": lse}
        if train:
            dh, dw = lm.cross_entropy_backward(s["grad"], s["hidden"], s["weight"], s["targets"], lse, total,
                                               reduction="mean", **how)
            out.update(dhidden=dh, dweight=dw)
        return out
    return _own_adamw(s)


# ------------------------------------------------------------------ 64 bits
def _exact_loss(s):
    c = s["case"]
    n, v, eps = c["tokens"], c["vocab"], c["smoothing"]
    h, w, t = s["hidden"].double(), s["weight"].double(), s["targets"]
    live = (t != IGNORE) & (t >= 0) & (t < v)
    count = max(1, int(live.sum()))
    rows, lse = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.empty(n, dtype=torch.float64, device="cuda")
    dh, dw = torch.empty_like(h), torch.zeros_like(w)
    step = max(1, (1 << 27) // v)
    for a in range(0, n, step):
        k = slice(a, min(n, a + step))
        z = h[k] @ w.t()
        lse[k] = torch.logsumexp(z, 1)
        want = torch.full_like(z, eps / v)                     # the distribution that the target stands for
        at = torch.nonzero(live[k])[:, 0]
        want[at, t[k][at]] += 1 - eps
        rows[k] = (lse[k] - (want * z).sum(1)) * live[k]
        if c["pass"] == "train":
            dz = (torch.softmax(z, 1) - want) * (live[k].double() / count)[:, None]
            dh[k] = dz @ w
            dw += dz.t() @ h[k]
    out = {"loss": rows.sum() / count, "rows": rows, "lse": lse}
    return {**out, "dhidden": dh, "dweight": dw} if c["pass"] == "train" else out


def _exact_values(code, scale, signed):
    c = code.cpu().numpy().astype("int64")
    k = scale.cpu().numpy().astype("int64").repeat(BLOCK) - 127
    mag, bias = (c & 127, 7) if signed else (c, 15)
    e, m = mag >> 4, mag & 15
    y = np.where(e > 0, np.ldexp(1.0 + m / 16.0, e - bias), np.ldexp(m / 16.0, 1 - bias))
    return np.ldexp(np.where(signed & (c > 127), -y, y), k)


def _exact_rounded(x, bits, signed):
    size = np.abs(x).reshape(-1, BLOCK)
    top = np.maximum(size.max(1), 1e-300)
    k = np.clip(np.ceil(np.log2(top * 16 / 31)), -126, 126)[:, None]
    y = np.ldexp(size, -k.astype("int64")).reshape(-1)
    low = -6 if signed else -14
    e = np.maximum(np.frexp(y)[1] - 1, low)
    unit = np.ldexp(1.0, e - 4)
    part = y / unit
    up = np.floor((part - np.floor(part)) * 65536) + bits >= 65536
    q = (np.floor(part) + up) * unit
    if not signed:
        q = np.where((x > 0) & (q == 0), 2.0 ** (low - 4), q)
    return np.ldexp(np.sign(x) * np.minimum(q, 31 / 16), k.astype("int64").repeat(BLOCK, 1).reshape(-1))


def _exact_adamw(s):
    small, t = s["case"]["bits"] == 8, s["step"]
    if small and s["p"].numel() > 1 << 25:
        return None                                            # minutes on the host
    b1, b2, lr = ADAM["beta1"], ADAM["beta2"], ADAM["lr"]
    p, g = s["p"].double().cpu().numpy(), s["g"].double().cpu().numpy()
    norm = np.sqrt((g ** 2).sum())
    if s["max_norm"] and norm > s["max_norm"]:
        g = g * (s["max_norm"] / norm)
    if small:
        m, v = _exact_values(s["m"], s["m_scale"], True), _exact_values(s["v"], s["v_scale"], False)
    else:
        m, v = s["m"].double().cpu().numpy(), s["v"].double().cpu().numpy()
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    p = p * (1 - lr * ADAM["weight_decay"]) - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + ADAM["eps"])
    if small:
        u = _random32(torch.arange(m.size), s["seed"], t).numpy()
        m, v = _exact_rounded(m, u & 0xFFFF, True), _exact_rounded(v, u >> 16, False)
    out = {"params": p, "m": m, "v": v}
    if s["max_norm"]:
        out["norm"] = norm
    return out


def exact(case, seed):
    s = prepare(case, seed)
    train = case.get("pass") == "train"
    if case["op"] == "loss":
        return _exact_loss(s)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    if case["op"] == "embed":
        out = {"out": s["table"].double()[s["tokens"]] * s["scale"]}
        if train:
            d = torch.zeros(s["table"].shape, dtype=torch.float64, device="cuda")
            out["dtable"] = d.index_add_(0, s["tokens"], s["dout"].double() * s["scale"])
        return out
    x, w = s["x"].double(), s["weight"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    sd = torch.sqrt(var + F32_EPS)
    out = {"y": (x - mean) / sd * w + s["bias"].double()}
    if train:
        dy, n = s["dy"].double(), x.shape[1]
        xhat = (x - mean) / sd
        g = dy * w
        out["dx"] = (n * g - g.sum(1, keepdim=True) - xhat * (g * xhat).sum(1, keepdim=True)) / (n * sd)
        out["dweight"], out["dbias"] = (dy * xhat).sum(0), dy.sum(0)
    return out


def work(case):
    """Bytes and operations that a pass cannot do without: each input read once, each output written once."""
    e = 2 if case.get("dtype") == "bf16" else 4
    train = case.get("pass") == "train"
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * (4 if train else 2) + case["cols"] * 4 * (4 if train else 2),
                "flops": n * (20 if train else 8)}
    if case["op"] == "embed":
        n = case["tokens"] * case["cols"]
        rows = min(case["tokens"], case["vocab"]) * case["cols"]
        return {"bytes": e * (n + rows) + 8 * case["tokens"] + (e * (n + case["vocab"] * case["cols"]) if train else 0),
                "flops": n * (2 if train else 1)}
    if case["op"] == "loss":
        n, d, v = case["tokens"], case["cols"], case["vocab"]
        return {"bytes": e * (n + v) * d * (2 if train else 1) + 16 * n, "flops": 2.0 * n * v * d * (3 if train else 1)}
    n = sum(_numels(case))
    moments = 4 + 4 if case["bits"] == 8 else 16           # read and written; the 8-bit ones' values too
    return {"bytes": n * (3 * e + moments), "flops": n * 15}
