"""Attention on the GPU, both passes, against the formulas in 64 bits.

Errors. A score is a sum of dim products: (dim + 8) roundings of scale sum |q||k|, the largest of which in a row is
`dz`. A probability's relative error is then at most twice that, and a rounding of each of its exponent's terms and of
the exponential; a sum over n terms adds n roundings of the terms' magnitudes. bfloat16 rounds p and ds once, 2^-8 of
each, and delta is formed from the rounded o. A probability below 2^-126, the smallest normal number, counts as zero
(exp2 gives no subnormal ones): that is off by less than 2^-126, whatever the rest.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from lm_check import U32, UNIT, slope, within  # noqa: E402
from paper_2310_12298_amd import lm  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")
TINY = 2.0 ** -126


def seen_by(nq, nk, tq, tk, causal, window):
    """(tq, tk) truth values: which keys a query sees."""
    i, j = torch.arange(tq)[:, None], torch.arange(tk)[None, :]
    seen = (i < nq) & (j < nk)
    if causal:
        at = nk - nq + i
        seen &= j <= at
        if window:
            seen &= j > at - window
    return seen


def plain(q, k, v, dout=None, scale=None, causal=False, window=None, ql=None, kl=None):
    """Results in 64 bits, and as "<name>_off" how far the call's may be before their own rounding."""
    dt = q.dtype
    q, k, v = (t.double().cpu() for t in (q, k, v))
    b, tq, h, d = q.shape
    tk, hk = k.shape[1], k.shape[2]
    g = h // hk
    scale = d ** -0.5 if scale is None else scale
    low = UNIT[dt] if dt is BF16 else 0.0
    names = ["out"] + (["dq", "dk", "dv"] if dout is not None else [])
    shapes = {"out": q, "dq": q, "dk": k, "dv": v}
    res = {n: torch.zeros_like(shapes[n]) for n in names}
    res.update({n + "_off": torch.zeros_like(shapes[n]) for n in names})
    res["lse"], res["lse_off"] = torch.full((b, h, tq), -INF).double(), torch.zeros(b, h, tq).double()
    for n in range(b):
        nq = tq if ql is None else min(max(int(ql[n]), 0), tq)
        nk = tk if kl is None else min(max(int(kl[n]), 0), tk)
        seen = seen_by(nq, nk, tq, tk, causal, window)
        rows = seen.any(1)
        if not rows.any():
            continue
        for m in range(h):
            x, y, w = q[n, rows, m], k[n, :nk, m // g], v[n, :nk, m // g]
            mask = seen[rows][:, :nk]
            z = scale * (x @ y.t())
            z[~mask] = -INF
            zs = scale * (x.abs() @ y.abs().t()) * mask
            lse = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[:, None])
            o = p @ w
            dz = (d + 8) * U32 * zs.max(1).values
            top = torch.where(mask, z.abs(), 0.0).max(1).values + lse.abs()
            rel = (2 * dz + U32 * (nk + 64 + 8 * top))[:, None]
            osize = p @ w.abs()
            ooff = osize * (rel + low) + TINY * (mask.double() @ w.abs())
            res["out"][n, rows, m], res["out_off"][n, rows, m] = o, ooff
            res["lse"][n, m, rows], res["lse_off"][n, m, rows] = lse, rel[:, 0]
            if dout is None:
                continue
            do = dout[n, rows, m].double().cpu()
            dp, delta = do @ w.t(), (do * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            dps = do.abs() @ w.abs().t()
            doff = (do.abs() * (ooff + UNIT[dt] * (o.abs() + ooff))).sum(1, keepdim=True)
            doff = doff + (d + 8) * U32 * (do.abs() * o.abs()).sum(1, keepdim=True)
            soff = p * (rel * (dp.abs() + delta.abs()) * (1 + rel) + (d + 8) * U32 * dps + doff)
            soff = soff + TINY * mask * (dp.abs() + delta.abs())
            soff = soff + (low + 4 * U32) * (ds.abs() + soff)
            poff = p * (rel + low * (1 + rel)) + TINY * mask
            for name, at, got, off, size, terms in (
                    ("dq", (n, rows, m), ds @ y, soff @ y.abs(), (ds.abs() + soff) @ y.abs(), nk),
                    ("dk", (n, slice(0, nk), m // g), ds.t() @ x, soff.t() @ x.abs(), (ds.abs() + soff).t() @ x.abs(), nq),
                    ("dv", (n, slice(0, nk), m // g), p.t() @ do, poff.t() @ do.abs(), (p + poff).t() @ do.abs(), nq)):
                f = 1.0 if name == "dv" else scale
                res[name][at] += f * got
                res[name + "_off"][at] += f * (off + U32 * (terms * g + 64) * size)
    return res


def inputs(b, tq, tk, h, hk, d, dtype, seed=0, s=1.0):
    g = torch.Generator().manual_seed(seed + 7 * tq + tk + 31 * d)
    return [(torch.randn(shape, generator=g) * s).to(dtype).cuda()
            for shape in ((b, tq, h, d), (b, tk, hk, d), (b, tk, hk, d), (b, tq, h, d))]


def check(q, k, v, dout, ql=None, kl=None, **how):
    lengths = {n: None if t is None else torch.as_tensor(t, device="cuda") for n, t in
               (("q_lengths", ql), ("kv_lengths", kl))}
    want = plain(q, k, v, dout, ql=ql, kl=kl, **how)
    out, lse = lm.attention_forward(q, k, v, **how, **lengths)
    assert out.shape == q.shape and out.dtype == q.dtype
    none = want["lse"] == -INF
    assert torch.equal(lse.cpu() == -INF, none)
    within(lse.cpu()[~none], want["lse"][~none], want["lse_off"][~none] / U32, 1, "lse")
    within(out, want["out"], want["out_off"] / U32, 1, "out")
    assert torch.count_nonzero(out.cpu().transpose(1, 2)[none]) == 0
    grads = lm.attention_backward(dout, q, k, v, out, lse, **how, **lengths)
    for n, t in zip(("dq", "dk", "dv"), grads):
        within(t, want[n], want[n + "_off"] / U32, 1, n)
    return out, lse, grads


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("b,tq,tk,h,hk,d", [
    (1, 1, 1, 1, 1, 64), (2, 1, 70, 4, 4, 64), (1, 1, 333, 8, 1, 128), (2, 3, 129, 6, 2, 40), (1, 31, 31, 1, 1, 8),
    (1, 33, 65, 2, 1, 128), (2, 64, 64, 2, 2, 64), (1, 65, 63, 3, 1, 72), (2, 127, 200, 4, 2, 128),
    (1, 129, 128, 2, 2, 1), (1, 200, 40, 2, 1, 33), (1, 300, 301, 3, 3, 127), (2, 257, 257, 4, 1, 96)])
def test_sizes(b, tq, tk, h, hk, d, dtype, causal):
    check(*inputs(b, tq, tk, h, hk, d, dtype), causal=causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 5000])
@pytest.mark.parametrize("tq,tk", [(1, 300), (150, 150), (70, 260), (260, 70)])
def test_windows(tq, tk, window, dtype):
    check(*inputs(1, tq, tk, 4, 2, 64, dtype), causal=True, window=window)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal,window", [(False, None), (True, None), (True, 40)])
def test_lengths(dtype, causal, window):
    """Whole, empty, single, odd ones, ones outside the range; of the keys, of the queries, of both."""
    some = [0, 1, 33, 64, 150, -3, 999]
    other = [150, 64, 7, 0, 1, 20, 149]
    q, k, v, dout = inputs(7, 150, 150, 4, 2, 72, dtype)
    for ql, kl in ((None, some), (some, None), (some, some), (other, some)):
        check(q, k, v, dout, ql, kl, causal=causal, window=window)
    q, k, v, dout = inputs(7, 3, 150, 4, 2, 72, dtype)
    check(q, k, v, dout, None, some, causal=causal, window=window)
    check(q, k, v, dout, [3, 0, 1, 2, 3, 1, 2], some, causal=causal, window=window)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tq,h,hk", [(37, 1, 1), (777, 6, 2), (1, 3, 1), (5, 2, 2)])
def test_an_empty_sequence_next_to_a_whole_one(tq, h, hk, dtype):
    """Rows of two sequences share a wave wherever heads and queries are odd."""
    q, k, v, dout = inputs(3, tq, 301, h, hk, 40, dtype)
    for kl in ([0, 301, 150], [150, 0, 301], [301, 150, 0]):
        check(q, k, v, dout, None, kl)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_keys_cut_into_ranges(dtype):
    """Few workgroups over many keys, and few keys under many queries: sums joined from ranges."""
    check(*inputs(1, 1, 9000, 8, 2, 128, dtype), causal=True)
    check(*inputs(2, 4, 5001, 2, 2, 64, dtype), kl=[5001, 700])
    check(*inputs(1, 100, 4000, 1, 1, 64, dtype), causal=True)
    check(*inputs(1, 3000, 90, 2, 1, 128, dtype))
    check(*inputs(1, 1000, 2500, 2, 1, 40, dtype), causal=True, window=900)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_far_apart(dtype):
    q, k, v, dout = inputs(1, 90, 200, 2, 1, 64, dtype, s=3.0)
    check(q, k, v, dout, scale=1.0, causal=True)
    check(q, k, v, dout, scale=1e-6)
    order = torch.argsort((q.float()[0, :, 0] @ k.float()[0, :, 0].t())[0])   # growing scores: every tile a new maximum
    check(q, k[:, order].contiguous(), v, dout, scale=0.7)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 40, 33])
def test_strides_and_alignment(d, dtype):
    q, k, v, dout = inputs(2, 77, 77, 6, 3, d, dtype)
    how = dict(causal=True)
    first = lm.attention_forward(q, k, v, **how)
    grads = lm.attention_backward(dout, q, k, v, *first, **how)
    n = q.shape[2] + 2 * k.shape[2]
    rows = torch.empty(2, 77, n, d, dtype=dtype, device="cuda")               # as one projection leaves them
    rows[:, :, :6], rows[:, :, 6:9], rows[:, :, 9:] = q, k, v
    turned = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v, dout)]
    odd = [torch.empty(t.numel() + 3, dtype=dtype, device="cuda")[3:].view(t.shape).copy_(t) for t in (q, k, v, dout)]
    dense = [t.permute(3, 0, 1, 2).contiguous().permute(1, 2, 3, 0) for t in (q, k, v, dout)]
    for a, b, c, g in ([rows[:, :, :6], rows[:, :, 6:9], rows[:, :, 9:], dout], turned, odd, dense):
        out = lm.attention_forward(a, b, c, **how)
        assert torch.equal(out[0], first[0]) and torch.equal(out[1], first[1])
        for x, y in zip(lm.attention_backward(g, a, b, c, *out, **how), grads):
            assert torch.equal(x, y)
    far = torch.zeros(2, 2, lm.ATTENTION_MAX_STRIDE + 8, dtype=dtype, device="cuda")
    far = far[:, :, :3 * d].unflatten(2, (3, d)).copy_(k[:, :2])
    assert torch.equal(lm.attention_forward(q, far, far)[0], lm.attention_forward(q, *(k[:, :2].contiguous(),) * 2)[0])
    one = dout[:, :1, :1].expand_as(dout)                                     # a broadcast gradient
    for x, y in zip(lm.attention_backward(one, q, k, v, *first, **how),
                    lm.attention_backward(one.contiguous(), q, k, v, *first, **how)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tq", [5, 150])
def test_what_stands_past_the_lengths_reaches_nothing(tq, dtype):
    q, k, v, dout = inputs(3, tq, 150, 4, 2, 64, dtype)
    ql, kl = [tq, 2, tq - 3], [100, 0, 77]
    lengths = dict(q_lengths=torch.tensor(ql, device="cuda"), kv_lengths=torch.tensor(kl, device="cuda"))
    for how in (dict(), dict(causal=True), dict(causal=True, window=30)):
        first = lm.attention_forward(q, k, v, **how, **lengths)
        grads = lm.attention_backward(dout, q, k, v, *first, **how, **lengths)
        for bad in (float("nan"), INF):
            Q, K, V, G = (t.clone() for t in (q, k, v, dout))
            for n in range(3):
                K[n, kl[n]:], V[n, kl[n]:], Q[n, ql[n]:], G[n, ql[n]:] = bad, bad, bad, bad
                if how:                                       # queries before the first key see nothing
                    Q[n, :max(0, ql[n] - kl[n])], G[n, :max(0, ql[n] - kl[n])] = bad, bad
            out = lm.attention_forward(Q, K, V, **how, **lengths)
            assert torch.equal(out[0], first[0]) and torch.equal(out[1], first[1])
            for x, y in zip(lm.attention_backward(G, Q, K, V, *out, **how, **lengths), grads):
                assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [24, 64, 96, 128])
@pytest.mark.parametrize("tq,window", [(3, None), (150, None), (150, 40), (400, 70)])
def test_nan_and_infinity_where_they_are_not_seen(tq, window, d, dtype):
    """Keys of the future, keys before the window, and gradients and queries of rows that do not see a key, in the same
    tile as those that do."""
    tk, how = 400, dict(causal=True, window=window)
    q, k, v, dout = inputs(1, tq, tk, 4, 2, d, dtype)
    off, first = tk - tq, tk - tq + 1 + tq // 3                # the first key of the future for the rows before `rows`
    rows = first - off
    want = plain(q, k, v, dout, **how)
    clean = lm.attention_forward(q, k, v, **how)
    grads = lm.attention_backward(dout, q, k, v, *clean, **how)

    def close(got, name, at):
        within(got[at], want[name][at], want[name + "_off"][at] / U32, 1, name)
    for bad in (float("nan"), INF, -INF):
        K, V = k.clone(), v.clone()
        K[:, first:, 0, 0], V[:, first:, 1, -1] = bad, bad
        gone = max(0, off - (window or tk))                    # keys that no query sees any more
        K[:, :gone], V[:, :gone] = bad, bad
        for a, b in ((K, v), (k, V), (K, V)):
            out, lse = lm.attention_forward(q, a, b, **how)
            assert torch.equal(lse[:, :, :rows], clean[1][:, :, :rows])
            close(out, "out", (slice(None), slice(0, rows)))
            dq = lm.attention_backward(dout, q, a, b, out, lse, need_kv=False, **how)[0]
            close(dq, "dq", (slice(None), slice(0, rows)))
        if not bool(torch.isfinite(torch.tensor(bad))) and rows < tq and V is not v:
            assert not bool(torch.isfinite(out[:, rows:].float()).all())
        Q, G = q.clone(), dout.clone()
        Q[:, :rows, 1], G[:, :rows, 2, 0] = bad, bad           # the rows before `rows` do not see the keys from `first` on
        for a, b in ((Q, dout), (q, G), (Q, G)):
            out, lse = lm.attention_forward(a, k, v, **how)
            for got, ref in zip(lm.attention_backward(b, a, k, v, out, lse, **how)[1:], grads[1:]):
                assert torch.equal(got[:, first:], ref[:, first:])
            for got, ref in zip(lm.attention_backward(b, a, k, v, out, lse, need_q=False, **how)[1:], grads[1:]):
                assert torch.equal(got[:, first:], ref[:, first:])
        seen = max(0, off + rows - (window or tk))             # a key that the last of them sees
        _, dk, dv = lm.attention_backward(G, q, k, v, *clean, **how)
        assert not bool(torch.isfinite(dv[0, max(seen, first - 1), 1].float()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tq", [2, 200])
def test_nan_and_infinity_where_they_are_seen(tq, dtype):
    q, k, v, dout = inputs(1, tq, 200, 2, 2, 64, dtype)
    clean = lm.attention_forward(q, k, v, causal=True)
    q[0, 1, 0] = float("nan")
    out, lse = lm.attention_forward(q, k, v, causal=True)
    assert bool(torch.isnan(out[0, 1, 0]).all()) and bool(torch.isnan(lse[0, 0, 1]))
    out[0, 1, 0], lse[0, 0, 1] = clean[0][0, 1, 0], clean[1][0, 0, 1]
    assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
    q, k, v, dout = inputs(1, tq, 200, 2, 2, 64, dtype)
    v[0, 5, 1] = INF
    out, lse = lm.attention_forward(q, k, v)
    assert torch.equal(lse, lm.attention_forward(q, k, v.clamp(max=9))[1])
    assert bool((out[0, :, 1] == INF).all()) and bool(torch.isfinite(out[0, :, 0]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nothing_to_do(dtype):
    for b, tq, tk in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        q, k, v, dout = inputs(b, tq, tk, 4, 2, 64, dtype)
        out, lse = lm.attention_forward(q, k, v)
        assert out.shape == q.shape and torch.count_nonzero(out) == 0 and bool((lse == -INF).all())
        for x, t in zip(lm.attention_backward(dout, q, k, v, out, lse), (q, k, v)):
            assert x.shape == t.shape and torch.count_nonzero(x) == 0
    q, k, v, dout = inputs(1, 40, 40, 4, 2, 64, dtype)
    out, lse = lm.attention_forward(q, k, v)
    every = lm.attention_backward(dout, q, k, v, out, lse)
    dq, dk, dv = lm.attention_backward(dout, q, k, v, out, lse, need_kv=False)
    assert torch.equal(dq, every[0]) and dk is None and dv is None
    dq, dk, dv = lm.attention_backward(dout, q, k, v, out, lse, need_q=False)
    assert dq is None and torch.equal(dk, every[1]) and torch.equal(dv, every[2])


def test_gradients_agree_with_differences_and_repeat_themselves():
    q, k, v, dout = inputs(2, 37, 50, 4, 2, 24, F32)
    kl = torch.tensor([50, 21], device="cuda")
    how = dict(causal=True, window=30)
    grads = []
    for _ in range(2):
        leaves = [t.clone().requires_grad_() for t in (q, k, v)]
        lm.attention(*leaves, **how, kv_lengths=kl).backward(dout)
        grads.append([t.grad for t in leaves])
    assert all(torch.equal(a, b) for a, b in zip(*grads))
    ref = [t.double().cpu() for t in (q, k, v)]
    seen = torch.stack([seen_by(37, int(n), 37, 50, True, 30) for n in kl.tolist()])[:, None]

    def loss(t):
        x, y, w = (a.transpose(1, 2) for a in t)
        y, w = y.repeat_interleave(2, 1), w.repeat_interleave(2, 1)
        z = (x @ y.transpose(2, 3) / 24 ** 0.5).masked_fill(~seen, -INF)
        p = torch.where(seen, torch.softmax(z, 3), 0.0).nan_to_num(0.0)
        return ((p @ w).transpose(1, 2) * dout.double().cpu()).sum()
    g = torch.Generator().manual_seed(1)
    for i, got in enumerate(grads[0]):
        d = torch.randn(ref[i].shape, generator=g, dtype=torch.float64)
        want = slope(lambda t: loss([t if j == i else r for j, r in enumerate(ref)]), ref[i], d, 1e-6)
        got = got.double().cpu()
        assert abs((got * d).sum() - want) <= 1e-5 * got.norm() * d.norm()


def test_autograd_of_some_inputs_and_a_shared_one():
    q, k, v, dout = inputs(1, 40, 40, 2, 2, 64, BF16)
    leaf = k.clone().requires_grad_()
    lm.attention(q, leaf, leaf, causal=True).backward(dout)
    out, lse = lm.attention_forward(q, k, k, causal=True)
    _, dk, dv = lm.attention_backward(dout, q, k, k, out, lse, causal=True)
    assert torch.equal(leaf.grad, dk + dv)
    leaf = q.clone().requires_grad_()
    lm.attention(leaf, k, v).backward(dout)
    assert leaf.grad is not None and torch.isfinite(leaf.grad).all()


def test_refusals():
    q, k, v, dout = inputs(2, 8, 8, 4, 2, 32, F32)
    out, lse = lm.attention_forward(q, k, v)
    n = torch.tensor([3, 4], device="cuda")
    for bad in (lambda: lm.attention_forward(q.half(), k.half(), v.half()), lambda: lm.attention_forward(q.cpu(), k, v),
                lambda: lm.attention_forward(q, k.bfloat16(), v.bfloat16()), lambda: lm.attention_forward(q, k, v[:, :7]),
                lambda: lm.attention_forward(q[:1], k, v), lambda: lm.attention_forward(q[..., :31], k, v),
                lambda: lm.attention_forward(q[:, :, :3], k, v), lambda: lm.attention_forward(q[0], k, v),
                lambda: lm.attention_forward(q, k, v, window=4), lambda: lm.attention_forward(q, k, v, True, window=0),
                lambda: lm.attention_forward(q, k, v, causal=True, window=0),
                lambda: lm.attention_forward(q, k, v, kv_lengths=n[:1]),
                lambda: lm.attention_forward(q, k, v, kv_lengths=n.float()),
                lambda: lm.attention_backward(dout[:, :7], q, k, v, out, lse),
                lambda: lm.attention_backward(dout.bfloat16(), q, k, v, out, lse),
                lambda: lm.attention_backward(dout, q, k, v, out, lse[:, :, :7])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lm.attention_forward(q, k, v, scale=0.0), lambda: lm.attention_forward(q, k, v, scale=-1.0),
                lambda: lm.attention_forward(q, k, v, scale=float("nan")),
                lambda: lm.attention_forward(*[torch.zeros(1, 1, 1, 129, device="cuda")] * 3)):
        with pytest.raises(lm.JorgeError):
            bad()


@pytest.mark.parametrize("batch,n,m,heads,kv_heads,dim,how", [
    (15, 2, 2, 8, 8, 94, dict(causal=True)), (7, 1809, 2, 7, 7, 53, {}), (4, 300, 300, 4, 2, 64, dict(causal=True, window=4)),
    (6, 96, 96, 8, 4, 80, dict(causal=True)), (3, 500, 21, 8, 2, 128, {})])
def test_bfloat16_gradients_where_rows_see_few_keys(batch, n, m, heads, kv_heads, dim, how):
    """dq and dk are rounded twice, each time by at most 2^-8 of a value, evenly: ds for its product and the result. The
    root mean square of that is 2^-8 / sqrt(3) at most, and that of both sqrt(2) times as much, 3.2e-3 of the result
    where the terms are independent. delta from the rounded o would add as much again where a row sees two keys."""
    g = torch.Generator().manual_seed(n + m + dim)
    q, dout = (torch.randn(batch, n, heads, dim, generator=g) for _ in range(2))
    k, v = (torch.randn(batch, m, kv_heads, dim, generator=g) for _ in range(2))
    q, k, v, dout = (t.bfloat16().cuda() for t in (q, k, v, dout))
    out, lse = lm.attention_forward(q, k, v, **how)
    Q, K, V = (t.double().requires_grad_() for t in (q, k, v))
    wide = [t.repeat_interleave(heads // kv_heads, 2).transpose(1, 2) for t in (K, V)]
    z = (Q.transpose(1, 2) @ wide[0].transpose(2, 3).contiguous()) * dim ** -0.5
    at = torch.arange(n, device="cuda")[:, None] + m - n
    key = torch.arange(m, device="cuda")[None]
    seen = torch.ones(n, m, dtype=torch.bool, device="cuda")
    if how:
        seen = (key <= at) & (key > at - how.get("window", m))
    z = torch.softmax(z.masked_fill(~seen, -float("inf")), -1)
    want = torch.autograd.grad((z @ wide[1]).transpose(1, 2), (Q, K, V), dout.double())
    for got, ref in zip(lm.attention_backward(dout, q, k, v, out, lse, **how)[:2], want):
        off = float((got.double() - ref).norm() / ref.norm())
        assert off < 2 ** 0.5 * 2 ** -8 / 3 ** 0.5, off


def test_many_sequences_over_long_caches_of_shared_heads():
    """64 sequences of 64 heads over 8: 2^27 rows counted with q's heads, 2^24 of k and v."""
    g = torch.Generator(device="cuda").manual_seed(5)
    q = torch.randn(64, 1, 64, 8, generator=g, device="cuda").bfloat16()
    k, v = (torch.randn(64, 32768, 8, 8, generator=g, device="cuda").bfloat16() for _ in range(2))
    kl = torch.randint(1, 32769, (64,), generator=g, device="cuda")
    out, lse = lm.attention_forward(q, k, v, causal=True, kv_lengths=kl)
    for n in (0, 41, 63):
        want = plain(q[n:n + 1], k[n:n + 1], v[n:n + 1], causal=True, kl=kl[n:n + 1])
        within(lse[n:n + 1], want["lse"], want["lse_off"] / U32, 1, "lse")
        within(out[n:n + 1], want["out"], want["out_off"] / U32, 1, "out")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_token_of_more_heads_than_a_token_stride_may_hold(dtype):
    """One token has no stride: 33000 heads of 128 are 4 224 000 elements apart from nothing."""
    q, k, v, dout = inputs(2, 1, 9, 33000, 1, 128, dtype)
    assert q.stride(1) > lm.ATTENTION_MAX_STRIDE
    out, lse = lm.attention_forward(q, k, v)
    grads = lm.attention_backward(dout, q, k, v, out, lse)
    few = [t[:, :, :64] for t in (q, dout)]
    part, part_lse = lm.attention_forward(few[0], k, v)
    assert torch.equal(lse[:, :64], part_lse) and torch.equal(out[:, :, :64], part)
    assert torch.equal(grads[0][:, :, :64], lm.attention_backward(few[1], few[0], k, v, part, part_lse)[0])


def test_long_sums_in_fp32_keep_their_precision():
    """A sum over n rows is formed tile by tile of 32: n / 32 roundings of the running sum, which grows with the root of
    the rows so far, make an error of at most 2^-24 sqrt(n / 64) of it. Backward a probability exp(z - lse) has the
    rounding of lse and that of lse log2(e) in it, 2^-24 lse each, and lse is at most log(keys) + 1 here. What a tile's own
    products, the scores and the exponentials add does not depend on n: e, measured where n is 256, and a tenth more.
    One by one the products would make 2^-24 sqrt(n / 4)."""
    def errors(nq, nk, hk, group):
        q, k, v, dout = inputs(1, nq, nk, hk * group, hk, 64, F32)
        out, lse = lm.attention_forward(q, k, v)
        got = [t[0].transpose(0, 1) for t in (out, *lm.attention_backward(dout, q, k, v, out, lse))]
        q, k, v, dout = (t[0].transpose(0, 1) for t in (q, k, v, dout))
        far, size = [0.0] * 4, [0.0] * 4
        for n in range(hk):
            K, V = k[n].double(), v[n].double()
            dk, dv = torch.zeros_like(K), torch.zeros_like(V)
            for m in range(n * group, (n + 1) * group):
                Q, G = q[m].double(), dout[m].double()
                p = torch.softmax(Q @ K.t() / 8, 1)
                o = p @ V
                ds = p * (G @ V.t() - (G * o).sum(1, keepdim=True)) / 8
                dk += ds.t() @ Q
                dv += p.t() @ G
                for i, want in ((0, o), (1, ds @ K)):
                    far[i] += float((got[i][m].double() - want).square().sum())
                    size[i] += float(want.square().sum())
            for i, want in ((2, dk), (3, dv)):
                far[i] += float((got[i][n].double() - want).square().sum())
                size[i] += float(want.square().sum())
        return [(a / b) ** 0.5 for a, b in zip(far, size)]
    e = [1.1 * x for x in errors(256, 256, 1, 4)]
    # Enough workgroups that neither axis is cut into ranges: of keys for out and dq, of queries for dk and dv.
    for nq, nk, hk, group, names in ((1024, 16384, 1, 64, ("out", "dq")), (4096, 1024, 64, 4, ("dk", "dv"))):
        every, lse = ("out", "dq", "dk", "dv"), 2 * (math.log(nk) + 1)
        for name, x, base in zip(every, errors(nq, nk, hk, group), e):
            n = nk if name in ("out", "dq") else nq * group
            room = (base ** 2 + U32 ** 2 * (n / 64 + (0 if name == "out" else lse) ** 2)) ** 0.5
            assert name not in names or x < room, f"{name} of {n} rows: {x:.2e}, room {room:.2e}"
