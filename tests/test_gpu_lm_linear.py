"""The linear layer and the gated projection on the GPU, both passes, against the formulas in 64 bits.

Roundings. A sum of K products takes at most K roundings of its accumulator in fp32, each relative to the sum of the
terms' magnitudes (products of bfloat16 are exact in fp32; three-term splits of fp32 take 6 K / 32, and leave out less
than three roundings of a product). An activation adds its own, at most 16, and carries its argument's error with its
slope, at most 1.13 (gelu's), its derivative with at most 0.8 (gelu's again). bfloat16: dz is rounded once before its
products, 2^-8 of each term.
"""
import pytest

torch = pytest.importorskip("torch")

from lm_check import U32, UNIT, slope, within  # noqa: E402
from paper_2310_12298_amd import lm  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")
SLOPE, BEND, OWN = 1.13, 0.8, 16
SIZES = [(1, 1, 1), (1, 33, 17), (3, 64, 128), (16, 100, 40), (17, 256, 65), (33, 515, 130), (64, 129, 96),
         (65, 64, 64), (70, 7, 300), (130, 1, 2), (200, 1023, 255), (257, 512, 513), (1025, 96, 320)]


def act64(name, z):
    if name is None:
        return z
    return {"relu": torch.relu, "gelu": lambda t: t * torch.special.ndtr(t), "silu": lambda t: t * torch.sigmoid(t),
            "sigmoid": torch.sigmoid}[name](z)


def both64(name, z):
    z = z.clone().requires_grad_()
    a = act64(name, z)
    return a.detach(), torch.autograd.grad(a.sum(), z)[0]


def rand(g, *shape, d, s=1.0):
    return (torch.randn(shape, generator=g) * s).to(d).cuda()


def check_linear(n, d, f, dtype, act, bias, residual, btype=F32):
    g = torch.Generator().manual_seed(n * 7 + d * 3 + f)
    x, w = rand(g, n, d, d=dtype), rand(g, f, d, d=dtype, s=d ** -0.5)
    b = rand(g, f, d=btype) if bias else None
    r = rand(g, n, f, d=dtype) if residual else None
    dy = rand(g, n, f, d=dtype)
    X, W, DY = (t.double().cpu() for t in (x, w, dy))
    B = b.double().cpu() if bias else torch.zeros(f, dtype=torch.float64)
    R = r.double().cpu() if residual else torch.zeros(n, f, dtype=torch.float64)
    zs = X.abs() @ W.abs().t() + B.abs()
    a, da = both64(act, X @ W.t() + B)
    y = lm.linear_forward(x, w, b, act, r)
    kz = d + OWN
    within(y, a + R, SLOPE * kz * zs + OWN * (a.abs() + zs) + 2 * R.abs(), 1, "y")
    dx, dw, db = lm.linear_backward(dy, x, w, b, act)
    dz = DY * da
    err = U32 * (DY.abs() * (BEND * kz * zs + OWN) if act else torch.zeros_like(dz))   # of dz, before its rounding
    rounded = UNIT[dtype] * dz.abs() if act and dtype is BF16 else 0
    for got, left, right, what in ((dx, lambda t: t, W, "dx"), (dw, lambda t: t.t(), X, "dweight")):
        terms = left(dz.abs() + err + rounded) @ right.abs()
        off = left(err + rounded) @ right.abs()
        within(got, left(dz) @ right, off / U32 + (left(dz).shape[1] + OWN) * terms, 1, what)
    if bias:
        within(db, dz.sum(0), err.sum(0) / U32 + (n + OWN) * dz.abs().sum(0), 1, "dbias")
        assert db.dtype == btype
    else:
        assert db is None


def check_gated(n, d, f, dtype, act):
    g = torch.Generator().manual_seed(n * 5 + d + f * 11)
    x, wg, wu = rand(g, n, d, d=dtype), rand(g, f, d, d=dtype, s=d ** -0.5), rand(g, f, d, d=dtype, s=d ** -0.5)
    dy = rand(g, n, f, d=dtype)
    X, G, U, DY = (t.double().cpu() for t in (x, wg, wu, dy))
    gs, us = X.abs() @ G.abs().t(), X.abs() @ U.abs().t()
    a, da = both64(act, X @ G.t())
    u = X @ U.t()
    kz = d + OWN
    y = lm.gated_linear_forward(x, wg, wu, act)
    within(y, a * u, SLOPE * kz * gs * u.abs() + (a.abs() + U32 * kz * gs) * kz * us + OWN * (a.abs() + gs) * us, 1, "y")
    dx, dg, du = lm.gated_linear_backward(dy, x, wg, wu, act)
    zg, zu = DY * u * da, DY * a
    eg = U32 * DY.abs() * (kz * us * (da.abs() + U32 * kz * gs) + us * (BEND * kz * gs + OWN))
    eu = U32 * DY.abs() * (SLOPE * kz * gs + OWN * (a.abs() + gs))
    low = UNIT[dtype] if dtype is BF16 else 0
    for e, z in ((eg, zg), (eu, zu)):
        e += low * (z.abs() + e)
    for got, z, e, what in ((dg, zg, eg, "dgate"), (du, zu, eu, "dup")):
        within(got, z.t() @ X, e.t() @ X.abs() / U32 + (n + OWN) * ((z.abs() + e).t() @ X.abs()), 1, what)
    terms = (zg.abs() + eg) @ G.abs() + (zu.abs() + eu) @ U.abs()
    within(dx, zg @ G + zu @ U, (eg @ G.abs() + eu @ U.abs()) / U32 + (2 * f + OWN) * terms, 1, "dx")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", SIZES)
def test_linear(n, d, f, dtype):
    check_linear(n, d, f, dtype, None, False, True)
    check_linear(n, d, f, dtype, "gelu", True, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", [None, "gelu", "silu", "sigmoid"])
@pytest.mark.parametrize("btype", [F32, BF16])
def test_linear_with_everything(dtype, act, btype):
    check_linear(150, 200, 333, dtype, act, True, True, btype)
    check_linear(9, 200, 333, dtype, act, True, True, btype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", SIZES)
def test_gated(n, d, f, dtype):
    check_gated(n, d, f, dtype, "silu")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", [None, "gelu", "sigmoid"])
def test_gated_activations(dtype, act):
    check_gated(140, 200, 333, dtype, act)
    check_gated(5, 200, 333, dtype, act)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", [(700, 2048, 640), (300, 4096, 200), (2048, 512, 2304)])
def test_products_cut_along_k_and_large_tiles(n, d, f, dtype):
    check_linear(n, d, f, dtype, "silu", True, True)
    check_gated(n, d, f, dtype, "silu")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", [(3000, 200, 6000), (6000, 4200, 330), (2050, 8200, 130)])
def test_the_largest_tiles(n, d, f, dtype):
    """Enough tiles of 256 x 256 for every CU, in each product; whole numbers, so every sum is exact."""
    g = torch.Generator().manual_seed(n)
    x, w, u, dy = whole(g, n, d, d=dtype), whole(g, f, d, d=dtype), whole(g, f, d, d=dtype), whole(g, n, f, d=dtype)
    X, W, U, DY = (t.double() for t in (x, w, u, dy))
    assert torch.equal(lm.linear_forward(x, w, None, "relu", dy), ((X @ W.t()).clamp(min=0) + DY).to(dtype))
    assert torch.equal(lm.gated_linear_forward(x, w, u, None), ((X @ W.t()) * (X @ U.t())).to(dtype))
    for act, dz in ((None, DY), ("relu", DY * (X @ W.t() > 0))):
        dx, dw, _ = lm.linear_backward(dy, x, w, None, act)
        assert torch.equal(dx, (dz @ W).to(dtype)) and torch.equal(dw, (dz.t() @ X).to(dtype))
    few = dy * (torch.rand(f, generator=g) < 8 / f).to(dtype).cuda()       # so that dg and du fit bfloat16's 8 bits
    x = x * (torch.rand(d, generator=g) < 6 / d).to(dtype).cuda()
    X, F = x.double(), few.double()
    dg, du = F * (X @ U.t()), F * (X @ W.t())
    assert float(dg.abs().max()) <= 256 and float(du.abs().max()) <= 256
    got = lm.gated_linear_backward(few, x, w, u, None)
    for a, c in zip(got, (dg @ W + du @ U, dg.t() @ X, du.t() @ X)):
        assert torch.equal(a, c.to(dtype))


def whole(g, *shape, d):
    """Small whole numbers, of which every product and sum here is exact."""
    return torch.randint(-2, 3, shape, generator=g).to(d).cuda()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [5, 90])
def test_relu_is_exact_and_has_no_slope_at_zero(n, dtype):
    g = torch.Generator().manual_seed(3)
    x, w, b, dy = whole(g, n, 24, d=dtype), whole(g, 40, 24, d=dtype), whole(g, 40, d=dtype), whole(g, n, 40, d=dtype)
    z = x.double() @ w.double().t() + b.double()
    assert bool((z == 0).any())
    dz = dy.double() * (z > 0)
    assert torch.equal(lm.linear_forward(x, w, b, "relu"), z.clamp(min=0).to(dtype))
    for a, c in zip(lm.linear_backward(dy, x, w, b, "relu"), (dz @ w.double(), dz.t() @ x.double(), dz.sum(0))):
        assert torch.equal(a, c.to(dtype))
    u = x.double() @ w.double().flip(0).t()
    z = x.double() @ w.double().t()
    assert torch.equal(lm.gated_linear_forward(x, w, w.flip(0), "relu"), (z.clamp(min=0) * u).to(dtype))


def test_activations_far_out():
    z = torch.tensor([-3e38, -1e4, -100.0, -89.0, -87.0, -20.0, 0.0, 20.0, 88.0, 1e4, 3e38, float("inf"),
                      float("nan")], device="cuda")
    one = torch.ones(1, 1, device="cuda")
    x = z[:, None]
    for n in (1, 9):                                      # few tokens, and (117 of them) many
        for act in ("silu", "gelu", "sigmoid", "relu"):
            y = lm.linear_forward(x.repeat(n, 1)[-117:], one, None, act)[-13:, 0]
            want = act64(act, z.double())
            finite = torch.isfinite(z)
            assert torch.allclose(y[finite].double(), want[finite], rtol=1e-5, atol=1e-5 * 21), (act, y)
            assert bool(torch.isnan(y[-1]))
            if n == 1:                                    # the splits know no infinity
                assert y[-2] == want[-2]
    dz = lm.linear_backward(torch.ones(11, 1, device="cuda"), x[:11], one, None, "silu")[0][:, 0]
    want = both64("silu", z[:11].double().cpu())[1]
    assert torch.allclose(dz.double().cpu(), want, atol=1e-6)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [40, 200])
def test_strided_rows_and_odd_starts(n, dtype):
    g = torch.Generator().manual_seed(11)
    d, f = 128, 192
    x, w, u, r, dy = (rand(g, a, b, d=dtype) for a, b in ((n, d), (f, d), (f, d), (n, f), (n, f)))

    def moved(t, start, more):
        hold = torch.full((start + t.shape[0] * (t.shape[1] + more),), float("nan"), dtype=dtype, device="cuda")
        v = hold[start:].view(t.shape[0], -1)[:, :t.shape[1]]
        v.copy_(t)
        return v
    first = [lm.linear_forward(x, w, None, "gelu", r), *lm.linear_backward(dy, x, w, None, "gelu")[:2],
             *lm.linear_backward(dy, x, w)[:2], lm.gated_linear_forward(x, w, u), *lm.gated_linear_backward(dy, x, w, u)]
    for start, more in ((0, 64), (1, 3), (8, 8)):
        X, W, U, R, D = (moved(t, start, more) for t in (x, w, u, r, dy))
        again = [lm.linear_forward(X, W, None, "gelu", R), *lm.linear_backward(D, X, W, None, "gelu")[:2],
                 *lm.linear_backward(D, X, W)[:2], lm.gated_linear_forward(X, W, U),
                 *lm.gated_linear_backward(D, X, W, U)]
        for i, (a, b) in enumerate(zip(first, again)):
            assert torch.equal(a, b), (start, i)
    # Turned weights, broadcast gradients and a row stride above what the call takes.
    wt = w.t().contiguous().t()
    assert torch.equal(lm.linear_forward(x, wt, None, "gelu", r), first[0])
    one = dy[:1].expand(n, f)
    for a, b in zip(lm.linear_backward(one, x, w)[:2], lm.linear_backward(one.contiguous(), x, w)[:2]):
        assert torch.equal(a, b)
    far = torch.zeros(2, lm.LINEAR_MAX_STRIDE + 8, dtype=dtype, device="cuda")[:, :d]
    far.copy_(x[:2])
    assert torch.equal(lm.linear_forward(far, w), lm.linear_forward(x[:2].contiguous(), w))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_tokens_and_single_gradients(dtype):
    g = torch.Generator().manual_seed(2)
    x, w, u, b, dy = (rand(g, *s, d=dtype) for s in ((0, 40), (72, 40), (72, 40), (72,), (0, 72)))
    assert lm.linear_forward(x, w, b, "silu").shape == (0, 72) and lm.gated_linear_forward(x, w, u).shape == (0, 72)
    for act in (None, "silu"):
        dx, dw, db = lm.linear_backward(dy, x, w, b, act)
        assert dx.shape == (0, 40) and torch.count_nonzero(dw) == 0 and torch.count_nonzero(db) == 0
    dx, dg, du = lm.gated_linear_backward(dy, x, w, u)
    assert dx.shape == (0, 40) and torch.count_nonzero(dg) == 0 and torch.count_nonzero(du) == 0
    x, dy = rand(g, 90, 40, d=dtype), rand(g, 90, 72, d=dtype)
    for act in (None, "gelu"):
        every = lm.linear_backward(dy, x, w, b, act)
        for k in range(3):
            need = [i == k for i in range(3)]
            got = lm.linear_backward(dy, x, w, b, act, *need)
            assert torch.equal(got[k], every[k]) and sum(t is None for t in got) == 2
        assert lm.linear_backward(dy, x, w, b, act, False, False, False) == (None, None, None)
    every = lm.gated_linear_backward(dy, x, w, u)
    assert torch.equal(lm.gated_linear_backward(dy, x, w, u, need_weights=False)[0], every[0])
    for a, c in zip(lm.gated_linear_backward(dy, x, w, u, need_x=False)[1:], every[1:]):
        assert torch.equal(a, c)


@pytest.mark.parametrize("n", [40, 200])
def test_a_row_of_nan_stays_alone(n):
    g = torch.Generator().manual_seed(4)
    for dtype in (F32, BF16):
        x, w, u, dy = (rand(g, *s, d=dtype) for s in ((n, 64), (96, 64), (96, 64), (n, 96)))
        clean = [lm.linear_forward(x, w, None, "gelu"), lm.gated_linear_forward(x, w, u),
                 lm.linear_backward(dy, x, w, None, "silu")[0], lm.gated_linear_backward(dy, x, w, u)[0]]
        x[7] = float("nan")
        got = [lm.linear_forward(x, w, None, "gelu"), lm.gated_linear_forward(x, w, u),
               lm.linear_backward(dy, x, w, None, "silu")[0], lm.gated_linear_backward(dy, x, w, u)[0]]
        keep = [i for i in range(n) if i != 7]
        for a, b in zip(got, clean):
            assert torch.equal(a[keep], b[keep]) and bool(torch.isnan(a[7]).all())


def test_gradients_agree_with_differences():
    g = torch.Generator().manual_seed(9)
    x, w, u, b, r, dy = (rand(g, *s, d=F32) for s in ((70, 33), (41, 33), (41, 33), (41,), (70, 41), (70, 41)))
    ref = [t.double().cpu() for t in (x, w, u, b, r)]
    DY = dy.double().cpu()

    def linear64(t):
        return ((act64("gelu", t[0] @ t[1].t() + t[3]) + t[4]) * DY).sum()

    def gated64(t):
        return (act64("silu", t[0] @ t[1].t()) * (t[0] @ t[2].t()) * DY).sum()
    for f64, call, which in ((linear64, lambda t: lm.linear(t[0], t[1], t[3], "gelu", t[4]), (0, 1, 3, 4)),
                             (gated64, lambda t: lm.gated_linear(t[0], t[1], t[2]), (0, 1, 2))):
        leaves = [t.clone().requires_grad_() for t in (x, w, u, b, r)]
        call(leaves).backward(dy)
        for k in which:
            v = torch.randn(ref[k].shape, generator=g, dtype=torch.float64)
            want = slope(lambda z: f64([z if i == k else t for i, t in enumerate(ref)]), ref[k], v, 1e-6)
            got = leaves[k].grad.double().cpu()
            assert abs((got * v).sum() - want) <= 1e-5 * got.norm() * v.norm(), k


def test_autograd_shapes_needs_and_the_same_bits_again():
    g = torch.Generator().manual_seed(12)
    x, w, u, b = (rand(g, *s, d=BF16).requires_grad_() for s in ((2, 3, 30, 64), (80, 64), (80, 64), (80,)))
    r = rand(g, 2, 3, 30, 80, d=BF16).requires_grad_()
    grads = []
    for _ in range(2):
        y = lm.linear(lm.gated_linear(x, w, u), torch.eye(80, dtype=BF16, device="cuda"), b, None, r)
        assert y.shape == r.shape
        y.square().sum().backward()
        grads.append([t.grad for t in (x, w, u, b, r)])
        for t in (x, w, u, b, r):
            t.grad = None
    assert all(torch.equal(p, q) for p, q in zip(*grads))
    y = lm.linear(x.detach(), w.detach(), b, "relu")
    y.sum().backward()
    assert b.grad is not None and x.grad is None


def test_outputs_past_two_to_the_31_elements():
    n, d, f = 70000, 16, 32768
    x = torch.zeros(n, d, dtype=BF16, device="cuda")
    x[-2:] = 1.0
    w = torch.zeros(f, d, dtype=BF16, device="cuda")
    w[-5:] = 2.0
    y = lm.linear_forward(x, w)
    assert bool((y[-2:, -5:] == 32).all()) and not bool(y[:-2].view(torch.int32).any())
    y = lm.gated_linear_forward(x, w, w, None)
    assert bool((y[-2:, -5:] == 1024).all()) and not bool(y[:-2].view(torch.int32).any())
    dx, dw, _ = lm.linear_backward(y, x, w)
    assert bool((dx[-2:] == 10240).all()) and bool((dw[-5:] == 2048).all()) and not bool(dw[:-5].any())


def test_refusals():
    g = torch.Generator().manual_seed(1)
    x, w, b, dy = (rand(g, *s, d=F32) for s in ((6, 32), (20, 32), (20,), (6, 20)))
    for bad in (lambda: lm.linear_forward(x.half(), w.half()), lambda: lm.linear_forward(x.cpu(), w),
                lambda: lm.linear_forward(x, w.bfloat16()), lambda: lm.linear_forward(x, w[:, :31]),
                lambda: lm.linear_forward(x, w, b[:19]), lambda: lm.linear_forward(x, w, activation="tanh"),
                lambda: lm.linear_forward(x, w, residual=dy[:5]), lambda: lm.linear_forward(x, w[0]),
                lambda: lm.linear_forward(x, w, residual=dy.bfloat16()),
                lambda: lm.linear_backward(dy[:, :19], x, w), lambda: lm.linear_backward(dy.bfloat16(), x, w),
                lambda: lm.gated_linear_forward(x, w, w[:19]), lambda: lm.gated_linear_forward(x, w, w.bfloat16()),
                lambda: lm.gated_linear_backward(dy[:5], x, w, w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(lm.JorgeError):
        lm.linear_forward(torch.zeros(1, 32769, device="cuda"), torch.zeros(1, 32769, device="cuda"))


@pytest.mark.parametrize("n,d,f,act", [(4096, 8192, 1536, None), (16384, 1030, 1100, None), (1500, 1000, 8192, "silu"),
                                       (700, 8192, 600, "silu")])
def test_long_sums_in_fp32_keep_their_precision(n, d, f, act):
    """A sum over K of random terms, and the step that it is rounded to, grow with the root of K, and so do the roundings'
    number and with it the sum's relative error, unless it is formed in ranges: their errors are independent and add up in
    squares as the ranges do, so that the whole errs as one range does. A range has 1024 terms up to K = 8192 (eight
    ranges), and K / 8 beyond. e is the error of a sum of 1024, measured. An argument's error e comes with the
    activation's slope: for silu of normal arguments, of act'(z) it is at most e (act'' is at most 1/2, the root mean
    square of act' 0.6) and of act(z) e (both have a root mean square of 0.6); and of u it is e. So a layer's gradients
    err by at most sqrt(2) e and the pair's by sqrt(3) e; a tenth more is left for what joins the ranges."""
    g = torch.Generator().manual_seed(n + d)
    x, w, u = (rand(g, *s, d=F32, s=k) for s, k in (((n, d), 1.0), ((f, d), d ** -0.5), ((f, d), d ** -0.5)))
    dy = rand(g, n, f, d=F32, s=1e-2)
    X, W, U, DY = (t.double() for t in (x, w, u, dy))

    def off(got, want):
        return float((got.double() - want).norm() / want.norm())

    a, b = rand(g, 4096, 1024, d=F32), rand(g, 4096, 1024, d=F32)      # enough tiles: its sums are of one range
    e = 1.1 * off(lm.linear_forward(a, b), a.double() @ b.double().t())

    def near(got, want, k, factor, what):
        assert off(got, want) < factor ** 0.5 * max(1.0, k / 8192) ** 0.5 * e, f"{what}: {off(got, want):.2e}, e {e:.2e}"

    a, da = both64(act, X @ W.t())
    more = 2 if act else 1
    near(lm.linear_forward(x, w, None, act), a, d, more, "y")
    dx, dw, _ = lm.linear_backward(dy, x, w, None, act)
    near(dx, DY * da @ W, f, more, "dx")
    near(dw, (DY * da).t() @ X, n, more, "dweight")
    if act:
        near(lm.gated_linear_forward(x, w, u, act), a * (X @ U.t()), d, 3, "gated y")
        dx, dw, du = lm.gated_linear_backward(dy, x, w, u, act)
        dg, dv = DY * (X @ U.t()) * da, DY * a
        near(dx, dg @ W + dv @ U, 2 * f, 3, "gated dx")
        near(dw, dg.t() @ X, n, 3, "dgate")
        near(du, dv.t() @ X, n, 3, "dup")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", [(130, 4001, 70), (70, 2500, 129), (300, 6000, 5)])
def test_few_tiles_of_long_rows(n, d, f, dtype):
    """Where K is cut over workgroups backward too, and dz is formed from the ranges' sums."""
    check_linear(n, d, f, dtype, "gelu", True, True)
    check_linear(n, d, f, dtype, "sigmoid", False, False)
    check_gated(n, d, f, dtype, "silu")


def test_single_gradients_of_few_tiles_of_long_rows():
    g = torch.Generator().manual_seed(4)
    x, w, u, b, dy = (rand(g, *s, d=F32) for s in ((130, 4001), (70, 4001), (70, 4001), (70,), (130, 70)))
    every = lm.linear_backward(dy, x, w, b, "silu")
    for i in range(3):
        alone = lm.linear_backward(dy, x, w, b, "silu", *[n == i for n in range(3)])
        assert torch.equal(alone[i], every[i]) and sum(t is not None for t in alone) == 1
    every = lm.gated_linear_backward(dy, x, w, u)
    assert torch.equal(lm.gated_linear_backward(dy, x, w, u, need_weights=False)[0], every[0])
    for one, both in zip(lm.gated_linear_backward(dy, x, w, u, need_x=False)[1:], every[1:]):
        assert torch.equal(one, both)


@pytest.mark.parametrize("tokens", [60, 2400])
def test_gelu_in_fp32_keeps_its_relative_precision(tokens):
    """gelu(z) = z Phi(z) is as small as Phi for z below 0, and its derivative Phi + z phi is their sum. A tail in fp32
    is off by 12 roundings of its polynomial, reciprocal and argument (evaluated on the host), 4 of the exponential and 2
    of a reciprocal that is one unit in the last place off; two more are the products'. Its argument and the matrix
    products are exact here (one column, weights of one)."""
    z = torch.linspace(-10, 4, 2400, device="cuda")
    z = z if tokens > lm.LINEAR_FEW_TOKENS else z[::40]
    x, one, zz = z[:, None].contiguous(), torch.ones(1, 1, device="cuda"), z.double().cpu()
    Phi, phi = 0.5 * torch.special.erfc(-zz / 2 ** 0.5), torch.exp(-0.5 * zz * zz) / (2 * torch.pi) ** 0.5
    within(lm.linear_forward(x, one, None, "gelu")[:, 0], zz * Phi, zz.abs() * Phi, 20, "gelu")
    within(lm.gated_linear_forward(x, one, one, "gelu")[:, 0], zz * zz * Phi, zz * zz * Phi, 21, "gated gelu")
    dx = lm.linear_backward(torch.ones_like(x), x, one, None, "gelu", need_weight=False)[0]
    within(dx[:, 0], Phi + zz * phi, Phi + zz.abs() * phi, 20, "gelu'")


def test_infinities_in_fp32_products_of_many_tokens():
    """An infinite element, or one that counts as such, makes infinities of the signs that the formula gives, and leaves
    all else as it is: as it does where few tokens are multiplied in fp32."""
    g = torch.Generator().manual_seed(6)
    n, d, f = 90, 40, 72
    x, w, u, dy = (rand(g, *s, d=F32) for s in ((n, d), (f, d), (f, d), (n, f)))
    clean = lm.linear_forward(x, w)
    few = [lm.linear_forward(x[:5], w), lm.linear_backward(dy, x, w)]
    for big in (INF, -INF, 3.4e38):
        for which in (x, w):
            a, b = x.clone(), w.clone()
            (a if which is x else b)[3, 7] = big
            y, want = lm.linear_forward(a, b), a.double() @ b.double().t()
            at = torch.zeros(n, f, dtype=torch.bool, device="cuda")
            at[(3,) if which is x else (slice(None), 3)] = True
            want = torch.sign(want) * INF
            assert torch.equal(y[at].double(), want[at]) and torch.equal(y[~at], clean[~at])
            if abs(big) == INF:
                y = lm.linear_forward(a[:5], b)
                assert torch.equal(y[at[:5]].double(), want[:5][at[:5]]) and torch.equal(y[~at[:5]], few[0][~at[:5]])
        G = dy.clone()
        G[11, 5] = big
        dx, dw, _ = lm.linear_backward(G, x, w)
        assert torch.equal(dx[11], torch.sign(w[5]) * big * INF) and torch.equal(dw[5], torch.sign(x[11]) * big * INF)
        for got, ref, row in ((dx, few[1][0], 11), (dw, few[1][1], 5)):
            keep = torch.arange(got.shape[0], device="cuda") != row
            assert torch.equal(got[keep], ref[keep])
    # With an activation: dz is split from the registers that formed it. u and g of the row are above 0 there.
    G, v = dy.clone(), x[11].sign() * w[5].abs() + 0.5 * x[11]
    w[5], u[5] = v, v
    ref = [lm.linear_backward(dy, x, w, None, "relu"), lm.gated_linear_backward(dy, x, w, u, "relu")]
    G[11, 5] = INF
    got = [lm.linear_backward(G, x, w, None, "relu"), lm.gated_linear_backward(G, x, w, u, "relu")]
    for a, b, rows in zip(got, ref, ((11, 5, None), (11, 5, 5))):
        for t, s, row in zip(a, b, rows):
            if t is not None:
                want = torch.sign(x[11] if row == 5 else w[5]) * INF
                assert torch.equal(t[row], want)
                keep = torch.arange(t.shape[0], device="cuda") != row
                assert torch.equal(t[keep], s[keep])


def test_memory_that_a_call_takes_beside_its_results():
    """None where bfloat16 operands are read as they lie and every product has a tile for each CU, so that no sum is cut; a
    frozen weight's gradient costs nothing in fp32 either."""
    g = torch.Generator(device="cuda").manual_seed(1)

    def beside(call):
        call()
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        out = call()
        after = torch.cuda.memory_allocated()
        torch.cuda.synchronize()
        return torch.cuda.max_memory_allocated() - after, sum(t is not None for t in out), after - before
    x, w, dy = (torch.randn(s, generator=g, device="cuda").to(BF16) for s in ((8192, 8192), (2048, 8192), (8192, 2048)))
    assert beside(lambda: (lm.linear_forward(x, w),))[0] == 0
    assert beside(lambda: lm.linear_backward(dy, x, w))[0] == 0
    x, w, dy = x.float(), w.float(), dy.float()
    every, dx = beside(lambda: lm.linear_backward(dy, x, w)), beside(lambda: lm.linear_backward(dy, x, w, need_weight=False))
    assert every[1] == 2 and dx[1] == 1
    assert every[0] - dx[0] > 6 * 8192 * (8192 + 2048) - 4 * 2048 * 8192
