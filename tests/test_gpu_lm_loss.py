"""Cross entropy over a vocabulary on the GPU, both passes, against the formula in 64 bits.

Room. A logit of `cols` products errs by at most (cols + 2) roundings of sum |h w| for bfloat16 inputs
(exact products, fp32 sums; the matrix unit adds 32 at a time, of which each counts) and, for fp32 ones,
by six such sums with the same bound; random signs leave it far below, so cols / 8 + 16 roundings of the
root of the sum of squares are allowed. The exponential adds |z - lse| roundings. lse takes the largest
logit's error and those of its own sum. Gradients: dz's own error (its rounding to bfloat16 for bfloat16
inputs: 2^-8 of each), as independent errors over the sum that they enter, five times over.
"""
import pytest

torch = pytest.importorskip("torch")

from lm_check import U32, UNIT, slope  # noqa: E402
from paper_2310_12298_amd import lm  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def inputs(n, d, v, dtype, seed=0, ignored=0.2, spread=2.0):
    g = torch.Generator().manual_seed(seed + n + 7 * d + 13 * v)
    h = torch.randn(n, d, generator=g).to(dtype)
    w = (torch.randn(v, d, generator=g) * (spread / d ** 0.5)).to(dtype)
    t = torch.randint(0, v, (n,), generator=g)
    t[torch.rand(n, generator=g) < ignored] = -100
    return h.cuda(), w.cuda(), t.cuda()


def plain(h, w, t, smoothing, ignore, row_grad):
    """Losses, lse, gradients and the errors to expect of them, on the GPU in 64 bits."""
    h, w = h.double(), w.double()
    v = w.shape[0]
    z = h @ w.t()
    lse = torch.logsumexp(z, 1)
    live = (t >= 0) & (t < v) & (t != ignore)
    want = torch.full_like(z, smoothing / v)
    at = torch.nonzero(live)[:, 0]
    want[at, t[at]] += 1 - smoothing
    loss = (lse - (want * z).sum(1)) * live
    g = row_grad(live) * live
    dz = (torch.softmax(z, 1) - want) * g[:, None]
    dz[~live] = 0
    zerr = ((h * h) @ (w * w).t()).sqrt() * (h.shape[1] / 8 + 16) * U32
    return dict(z=z, lse=lse, loss=loss, live=live, g=g, dz=dz, dh=dz @ w, dw=dz.t() @ (h * live[:, None]), zerr=zerr,
                p=torch.softmax(z, 1))


def close(got, want, room, what):
    got = got.double()
    assert got.shape == want.shape and bool(torch.isfinite(got).all()), what
    bad = ((got - want).abs() > room).nonzero()
    at = tuple(bad[0].tolist()) if len(bad) else None
    assert at is None, (what, len(bad), at, got[at].item(), want[at].item(), room.expand_as(want)[at].item())


def check(h, w, t, smoothing=0.0, ignore=-100, reduction="mean"):
    dtype, (n, d), v = h.dtype, h.shape, w.shape[0]
    gen = torch.Generator().manual_seed(1)
    per_row = torch.randn(n, generator=gen).cuda()
    one = torch.tensor(1.7, device="cuda")
    row_grad = {"none": lambda live: per_row.double(),
                "sum": lambda live: torch.full_like(live, 1.7, dtype=torch.float64),
                "mean": lambda live: 1.7 / live.sum().clamp(min=1) * live.double()}[reduction]
    want = plain(h, w, t, smoothing, ignore, row_grad)
    loss, lse, total = lm.cross_entropy_forward(h, w, t, ignore, smoothing)
    zroom = want["zerr"].max(1).values + want["z"].abs().max(1).values * 8 * U32
    lse_room = zroom + (want["lse"].abs() + 16) * 8 * U32
    close(lse, want["lse"], lse_room, "lse")
    close(loss, want["loss"], (2 * lse_room + want["z"].abs().max(1).values * v ** 0.5 * smoothing * 8 * U32), "loss")
    count = int(want["live"].sum())
    assert total[1].item() == count
    sums = want["loss"].sum()
    room = (2 * lse_room).sum() + sums.abs() * 4 * U32
    assert abs(total[0].item() - sums) <= room and abs(total[2].item() - sums / max(count, 1)) <= room / max(count, 1)
    back = (per_row if reduction == "none" else one, h, w, t, lse, total, reduction, ignore, smoothing)
    dh, dw = lm.cross_entropy_backward(*back)
    assert dh.dtype == dtype and dw.dtype == dtype
    # Errors of dz: those of p, and the rounding of each to the type that the products take.
    rel = want["zerr"] + lse_room[:, None] + (want["z"] - want["lse"][:, None]).abs() * 2 * U32 + 4 * U32
    err = want["p"] * want["g"].abs()[:, None] * rel + want["dz"].abs() * (UNIT[BF16] if dtype == BF16 else 4 * U32)
    e2 = err.square()
    hd, wd, live = h.double(), w.double(), want["live"]
    hl = hd * live[:, None]
    for got, ref, room2, terms in ((dh, want["dh"], e2 @ wd.square(), want["dz"].abs() @ wd.abs()),
                                   (dw, want["dw"], e2.t() @ hl.square(), want["dz"].abs().t() @ hl.abs())):
        room = 5 * room2.sqrt() + 40 * U32 * terms
        close(got, ref, room + UNIT[dtype] * (ref.abs() + room) + 1e-30, "gradient")
    assert torch.count_nonzero(dh[~live]) == 0
    again = lm.cross_entropy_backward(*back)
    assert torch.equal(again[0], dh) and torch.equal(again[1], dw)           # the same bits again


SIZES = [(1, 1, 1), (1, 8, 2), (3, 5, 7), (2, 64, 130), (63, 64, 64), (65, 70, 129), (128, 128, 128), (129, 257, 255),
         (200, 192, 513), (257, 320, 1000), (40, 1000, 3000), (1000, 48, 90), (5, 2048, 5000)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,v", SIZES)
def test_sizes(n, d, v, dtype):
    check(*inputs(n, d, v, dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_reductions_and_smoothing(reduction, smoothing, dtype):
    check(*inputs(150, 96, 700, dtype), smoothing=smoothing, reduction=reduction)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_tiles(dtype):
    check(*inputs(2100, 128, 4200, dtype))                   # 256 x 256 tiles of logits, odd edges both ways
    check(*inputs(4100, 4096, 300, dtype, spread=1.0))       # large tiles of both gradients


def test_several_pieces_of_the_vocabulary():
    check(*inputs(4000, 64, 50001, BF16))
    check(*inputs(3000, 100, 30011, F32), smoothing=0.1)


def test_few_words_many_tokens_cut_the_sum_over_tokens():
    check(*inputs(20000, 64, 40, BF16))
    check(*inputs(5000, 30, 17, F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_without_a_target(dtype):
    h, w, t = inputs(70, 64, 100, dtype, ignored=0.0)
    t[:] = -100
    loss, lse, total = lm.cross_entropy_forward(h, w, t)
    assert torch.count_nonzero(loss) == 0 and total.tolist() == [0.0, 0.0, 0.0]
    dh, dw = lm.cross_entropy_backward(torch.ones((), device="cuda"), h, w, t, lse, total)
    assert torch.count_nonzero(dh) == 0 and torch.count_nonzero(dw) == 0
    t = torch.randint(0, 100, (70,), device="cuda")
    t[::3] = 5
    check(h, w, t, ignore=5)                                 # a word of the vocabulary that is not counted
    t[1::3], t[2] = 100, 1 << 40                             # outside: no target either
    check(h, w, t)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nan_and_infinity_in_masked_rows_reach_nothing(dtype):
    h, w, t = inputs(90, 72, 300, dtype, ignored=0.0)
    t[[3, 50]] = -100
    out = []
    for fill in (0.0, float("nan"), float("inf")):
        h[3], h[50, 7] = fill, fill
        loss, lse, total = lm.cross_entropy_forward(h, w, t)
        out.append([loss, total, *lm.cross_entropy_backward(torch.ones((), device="cuda"), h, w, t, lse, total)])
    for other in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(out[0], other))


def test_large_logits_do_not_overflow():
    h, w, t = inputs(40, 64, 200, F32, spread=400.0)
    check(h, w, t)
    t[:] = (h @ w.t()).argmin(1)
    loss = lm.cross_entropy_forward(h, w, t)[0]
    assert bool((loss > 500).all()) and bool(torch.isfinite(loss).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_odd_starts(dtype):
    n, d, v = 70, 64, 150
    h, w, t = inputs(n, d, v, dtype)
    loss, lse, total = lm.cross_entropy_forward(h, w, t)
    grads = lm.cross_entropy_backward(torch.ones((), device="cuda"), h, w, t, lse, total)
    for ld, start in ((64, 1), (67, 0), (72, 8), (80, 3)):
        hh, hw = (torch.full((r * ld + start,), float("nan"), dtype=dtype, device="cuda") for r in (n, v))
        vh, vw = hh[start:].view(n, ld)[:, :d], hw[start:].view(v, ld)[:, :d]
        vh.copy_(h)
        vw.copy_(w)
        got = lm.cross_entropy_forward(vh, vw, t)
        assert all(torch.equal(a, b) for a, b in zip(got, (loss, lse, total)))
        got = lm.cross_entropy_backward(torch.ones((), device="cuda"), vh, vw, t, lse, total)
        assert all(torch.equal(a, b) for a, b in zip(got, grads))


def test_no_tokens():
    h, w = torch.empty(0, 16, device="cuda"), torch.ones(5, 16, device="cuda")
    t = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse, total = lm.cross_entropy_forward(h, w, t)
    assert loss.shape == (0,) and total.tolist() == [0.0, 0.0, 0.0]
    dh, dw = lm.cross_entropy_backward(torch.ones((), device="cuda"), h, w, t, lse, total)
    assert dh.shape == (0, 16) and torch.count_nonzero(dw) == 0 and dw.shape == (5, 16)


def test_autograd_and_differences():
    h, w, t = inputs(12, 20, 33, F32)
    h3 = h.view(3, 4, 20).requires_grad_()
    w = w.requires_grad_()
    for reduction in ("mean", "sum", "none"):
        h3.grad = w.grad = None
        out = lm.linear_cross_entropy(h3, w, t.view(3, 4), label_smoothing=0.1, reduction=reduction)
        assert out.shape == ((3, 4) if reduction == "none" else ())
        out.sum().backward()
        hd, wd, tc = h.detach().double(), w.detach().double(), t

        def f(a, b):
            x = plain(a, b, tc, 0.1, -100, lambda live: torch.ones_like(live, dtype=torch.float64))
            return x["loss"].sum() / (x["live"].sum() if reduction == "mean" else 1)
        gen = torch.Generator().manual_seed(2)
        u = torch.randn(12, 20, generator=gen, dtype=torch.float64).cuda()
        v = torch.randn(33, 20, generator=gen, dtype=torch.float64).cuda()
        want = slope(lambda x: f(x, wd), hd, u, 1e-5) + slope(lambda x: f(hd, x), wd, v, 1e-5)
        got = (h3.grad.view(12, 20).double() * u).sum() + (w.grad.double() * v).sum()
        assert abs(got - want) <= 1e-5 * (h3.grad.double().norm() * u.norm() + w.grad.double().norm() * v.norm())
    w.requires_grad_(False)
    h3.grad = None
    lm.linear_cross_entropy(h3, w, t.view(3, 4)).backward()   # one gradient alone
    assert h3.grad is not None and w.grad is not None


def test_refusals():
    h, w, t = inputs(8, 16, 30, F32)
    for bad in (lambda: lm.cross_entropy_forward(h, w.bfloat16(), t), lambda: lm.cross_entropy_forward(h, w[:, :15], t),
                lambda: lm.cross_entropy_forward(h, w, t[:7]), lambda: lm.cross_entropy_forward(h, w, t.float()),
                lambda: lm.cross_entropy_forward(h.half(), w.half(), t),
                lambda: lm.linear_cross_entropy(h, w, t, reduction="max")):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(lm.JorgeError):
        lm.cross_entropy_forward(h, w, t, label_smoothing=1.5)
    loss, lse, total = lm.cross_entropy_forward(h, w, t)
    with pytest.raises(ValueError):
        lm.cross_entropy_backward(torch.ones(3, device="cuda"), h, w, t, lse, total, reduction="none")
