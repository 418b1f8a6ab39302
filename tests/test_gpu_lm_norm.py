"""Layer norm on the GPU, both passes, against the formula in 64 bits.

Roundings: a lane adds at most 64 elements of a row one after the other, then six exchanges and
eight waves: 80 roundings of a sum over the terms' magnitudes, and a dozen of the element's own.
The gradients of gain and bias add rows / 768 (at least 1) rows by the lane, then at most 48 partial
sums by the wave, and sixteen waves. The mean's own error enters every element: 100 in all.
"""
import pytest

torch = pytest.importorskip("torch")

from lm_check import slope, within  # noqa: E402
from paper_2310_12298_amd import lm  # noqa: E402

pytestmark = pytest.mark.gpu
R = 100
F32, BF16 = torch.float32, torch.bfloat16


def plain(x, w, b, eps, dy=None):
    x, w, b = x.double(), w.double(), b.double()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    xh = c * r
    out = {"y": xh * w + b, "mean": mean[:, 0], "rstd": r[:, 0]}
    # How large the terms are: what a rounding is relative to.
    xs = (x.abs() + x.abs().mean(1, keepdim=True)) * r
    out["ysize"] = xs * w.abs() + b.abs()
    if dy is not None:
        dy = dy.double()
        g = dy * w
        m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
        out["dx"] = r * (g - m1 - xh * m2)
        s1, s2 = g.abs().mean(1, keepdim=True), (g.abs() * xs).mean(1, keepdim=True)
        out["dxsize"] = r * (g.abs() + s1 + xs * s2 * 2)
        out["dw"], out["db"] = (dy * xh).sum(0), dy.sum(0)
        out["dwsize"], out["dbsize"] = (dy.abs() * xs).sum(0), dy.abs().sum(0)
    return out


def inputs(rows, cols, dtype, ptype, seed=0):
    g = torch.Generator().manual_seed(seed + 31 * rows + cols)
    x = torch.randn(rows, cols, generator=g) * (0.2 + torch.rand(rows, 1, generator=g))
    x += torch.randn(rows, 1, generator=g)
    return [t.to(d).cuda() for t, d in ((x, dtype), (1 + 0.2 * torch.randn(cols, generator=g), ptype),
                                        (0.3 * torch.randn(cols, generator=g), ptype),
                                        (torch.randn(rows, cols, generator=g), dtype))]


def check(x, w, b, dy, eps=1e-5):
    want = plain(x.cpu(), w.cpu(), b.cpu(), eps, dy.cpu())
    y, mean, rstd = lm.layer_norm_forward(x, w, b, eps)
    assert y.dtype == x.dtype and y.shape == x.shape
    within(y, want["y"], want["ysize"], R, "y")
    within(mean, want["mean"], x.double().abs().mean(1), R, "mean")
    dx, dw, db = lm.layer_norm_backward(dy, x, mean, rstd, w)
    within(dx, want["dx"], want["dxsize"], R, "dx")
    within(dw, want["dw"], want["dwsize"], R, "dweight")
    within(db, want["db"], want["dbsize"], R, "dbias")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ptype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 2), (3, 7), (5, 64), (7, 255), (9, 257), (130, 512), (33, 1023), (2, 1025),
                                       (19, 2048), (800, 2049), (17, 4096), (3, 5001), (11, 8192), (5, 12289),
                                       (2, 16384)])
def test_both_passes(rows, cols, dtype, ptype):
    check(*inputs(rows, cols, dtype, ptype))


def test_many_rows_reach_every_partial_sum():
    check(*inputs(4001, 72, F32, F32))
    check(*inputs(2303, 1100, BF16, F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_single_column_is_its_bias(dtype):
    x, w, b, dy = inputs(6, 1, dtype, F32)
    y, mean, rstd = lm.layer_norm_forward(x, w, b)
    assert torch.equal(y, b.to(dtype).expand(6, 1))
    dx, dw, db = lm.layer_norm_backward(dy, x, mean, rstd, w)
    assert torch.count_nonzero(dx) == 0 and torch.count_nonzero(dw) == 0
    within(db, dy.double().sum(0), dy.double().abs().sum(0), R, "dbias")


def test_rows_far_from_zero_keep_their_variance():
    x, w, b, dy = inputs(4, 1000, F32, F32)
    x = x + 1e4                                        # squares of x would lose all of it
    check(x, w, b, dy)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strided_rows_and_odd_starts(dtype):
    for cols, ld, start in ((100, 133, 1), (1001, 1003, 3), (2000, 4096, 7)):
        x, w, b, dy = inputs(9, cols, dtype, F32)
        hx, hd = (torch.full((9 * ld + start,), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        vx, vd = (h[start:].view(9, ld)[:, :cols] for h in (hx, hd))
        vx.copy_(x)
        vd.copy_(dy)
        y, mean, rstd = lm.layer_norm_forward(vx, w, b)
        y0, m0, r0 = lm.layer_norm_forward(x, w, b)
        assert torch.equal(y, y0) and torch.equal(mean, m0) and torch.equal(rstd, r0)
        for a, c in zip(lm.layer_norm_backward(vd, vx, mean, rstd, w), lm.layer_norm_backward(dy, x, mean, rstd, w)):
            assert torch.equal(a, c)


def test_no_rows_no_gain_no_sums():
    x, w, b, dy = inputs(0, 40, F32, F32)
    y, mean, rstd = lm.layer_norm_forward(x, w, b)
    dx, dw, db = lm.layer_norm_backward(dy, x, mean, rstd, w)
    assert y.shape == (0, 40) and dx.shape == (0, 40)
    assert torch.count_nonzero(dw) == 0 and torch.count_nonzero(db) == 0
    x, w, b, dy = inputs(12, 40, F32, F32)
    ones, zeros = torch.ones_like(w), torch.zeros_like(b)
    y, mean, rstd = lm.layer_norm_forward(x)
    assert torch.equal(y, lm.layer_norm_forward(x, ones, zeros)[0])
    dx, dw, db = lm.layer_norm_backward(dy, x, mean, rstd)
    for a, c in zip((dx, dw, db), lm.layer_norm_backward(dy, x, mean, rstd, ones)):
        assert torch.equal(a, c)
    assert lm.layer_norm_backward(dy, x, mean, rstd, affine=False)[1:] == (None, None)
    assert torch.equal(lm.layer_norm_backward(dy, x, mean, rstd, affine=False)[0], dx)


def test_a_row_of_nan_or_infinity_stays_alone():
    x, w, b, dy = inputs(9, 300, F32, F32)
    clean = lm.layer_norm_forward(x, w, b)[0]
    x[4, 17] = float("inf")
    x[6, 0] = float("nan")
    y = lm.layer_norm_forward(x, w, b)[0]
    keep = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(y[keep], clean[keep]) and bool(torch.isnan(y[[4, 6]]).all())


def test_gradient_agrees_with_differences():
    x, w, b, dy = inputs(6, 129, F32, F32)
    x, w, b = x.requires_grad_(), w.requires_grad_(), b.requires_grad_()
    lm.layer_norm(x, w, b).backward(dy)
    g = torch.Generator().manual_seed(5)
    ref = [t.detach().double().cpu() for t in (x, w, b)]
    loss = lambda ts: (plain(*ts, 1e-5)["y"] * dy.double().cpu()).sum()  # noqa: E731
    for k, t in enumerate((x, w, b)):
        v = torch.randn(t.shape, generator=g, dtype=torch.float64)
        want = slope(lambda z: loss([z if i == k else r for i, r in enumerate(ref)]), ref[k], v, 1e-6)
        got = (t.grad.double().cpu() * v).sum()
        assert abs(got - want) <= 1e-5 * t.grad.double().norm().cpu() * v.norm()


def test_autograd_shapes_and_the_same_bits_again():
    x, w, b, dy = inputs(24, 96, BF16, F32)
    x3 = x.view(2, 3, 4, 96).requires_grad_()
    y = lm.layer_norm(x3, w.requires_grad_(), b.requires_grad_())
    y.backward(dy.view_as(x3))
    assert y.shape == x3.shape and x3.grad.shape == x3.shape
    first = [x3.grad.clone(), w.grad.clone(), b.grad.clone()]
    x3.grad = w.grad = b.grad = None
    lm.layer_norm(x3, w, b).backward(dy.view_as(x3))
    for a, c in zip(first, (x3.grad, w.grad, b.grad)):
        assert torch.equal(a, c)


def test_on_a_stream_of_its_own():
    x, w, b, dy = inputs(64, 768, F32, F32)
    torch.cuda.synchronize()
    want = lm.layer_norm_forward(x, w, b)[0]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = lm.layer_norm_forward(x, w, b)[0]
    s.synchronize()
    assert torch.equal(got, want)


def test_refusals():
    x, w, b, dy = inputs(4, 32, F32, F32)
    y, mean, rstd = lm.layer_norm_forward(x, w, b)
    for bad in (lambda: lm.layer_norm_forward(x.half()), lambda: lm.layer_norm_forward(x.cpu()),
                lambda: lm.layer_norm_forward(x, w[:31]), lambda: lm.layer_norm_forward(x, w, b.bfloat16()),
                lambda: lm.layer_norm_backward(dy.bfloat16(), x, mean, rstd, w),
                lambda: lm.layer_norm_backward(dy[:3], x, mean, rstd, w),
                lambda: lm.layer_norm_backward(dy, x, mean[:3], rstd, w)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lm.layer_norm_forward(x, eps=-1.0), lambda: lm.layer_norm_forward(x, eps=float("nan")),
                lambda: lm.layer_norm_forward(torch.zeros(1, 16385, device="cuda"))):
        with pytest.raises(lm.JorgeError):
            bad()
