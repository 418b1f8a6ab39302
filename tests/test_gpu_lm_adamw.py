"""AdamW and the global gradient norm on the GPU against the formulas in 64 bits.

Roundings of a 32-bit step: three of each moment (difference, product, sum) and the constant's own;
of the weight, those of the update (moment, rate, square root, two products, sum, quotient: a dozen,
relative to the update and the decay) and one to its type. The norm: 256 squares by the lane, the
rest in fp64.
"""
import io
import math

import pytest

torch = pytest.importorskip("torch")
np = pytest.importorskip("numpy")

from lm_check import U32, UNIT, within  # noqa: E402
from paper_2310_12298_amd import lm  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
HP = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
SIZES = [1, 255, 256, 257, 1000, 4096, 4097, 20000, 3, 70001]


def tensors(sizes, dtype, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * scale).to(dtype).cuda() for n in sizes]


def formula(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, clip=1.0):
    """New (p, m, v) in 64 bits, and the sizes of the terms that make up m, v and p's change."""
    g = g * clip
    m1, v1 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    u = lr * (m1 / (1 - beta1 ** t)) / (torch.sqrt(v1 / (1 - beta2 ** t)) + eps)
    usize = lr * ((m.abs() + g.abs()) / (1 - beta1 ** t)) / (torch.sqrt(v1 / (1 - beta2 ** t)) + eps)
    return p * (1 - lr * weight_decay) - u, m1, v1, m.abs() + g.abs(), v + g * g, usize + lr * weight_decay * p.abs()


def flat(opt, xs):
    out = torch.zeros(int(opt.blocks[-1]) * lm.BLOCK, dtype=torch.float64)
    for b, x in zip(opt.blocks, xs):
        out[b * lm.BLOCK: b * lm.BLOCK + x.numel()] = x.double().cpu().reshape(-1)
    return out


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("clip", [False, True])
def test_steps_in_32_bits(dtype, clip):
    params = tensors(SIZES, dtype)
    opt = lm.AdamW(params)
    for t in range(1, 4):
        grads = tensors(SIZES, dtype, seed=t, scale=0.1 * t)
        p, g = flat(opt, params), flat(opt, grads)
        m, v = (x.double().cpu() for x in opt.moment_values())
        norm = math.sqrt((g * g).sum())
        opt.step(grads, max_norm=0.5 * norm if clip else 0.0, **HP)
        assert opt.t == t
        # The clip factor's own roundings (norm, quotient) count as one more of each gradient.
        p1, m1, v1, ms, vs, ps = formula(p, g, m, v, t, clip=0.5 if clip else 1.0, **HP)
        got_m, got_v = opt.moment_values()
        within(got_m, m1, ms, 6, "m")
        within(got_v, v1, vs, 8, "v")
        for i, (q, b) in enumerate(zip(params, opt.blocks)):
            s = slice(b * lm.BLOCK, b * lm.BLOCK + q.numel())
            within(q, p1[s], ps[s], 24, f"p{i}")
        if clip:
            assert abs(opt.norm.item() - norm) <= 140 * U32 * norm


def test_norm_and_factor():
    opt = lm.AdamW(tensors(SIZES, F32))
    grads = tensors(SIZES, F32, seed=9)
    want = math.sqrt(sum((g.double() ** 2).sum().item() for g in grads))
    norm, f = opt.gradient_norm(grads, max_norm=1.0).tolist()
    assert abs(norm - want) <= 140 * U32 * want and abs(f - 1 / want) <= 150 * U32 / want
    assert opt.gradient_norm(grads).tolist()[1] == 1.0
    assert opt.gradient_norm(grads, max_norm=2 * want).tolist()[1] == 1.0
    assert opt.gradient_norm([torch.zeros_like(g) for g in grads], max_norm=1.0).tolist() == [0.0, 1.0]
    grads[3][100] = float("nan")
    assert all(math.isnan(x) for x in opt.gradient_norm(grads, max_norm=1.0).tolist())
    mixed = lm.AdamW(tensors([300], F32) + tensors([500], BF16))
    g = tensors([300], F32, seed=2) + tensors([500], BF16, seed=3)
    want = math.sqrt(sum((x.double() ** 2).sum().item() for x in g))
    assert abs(mixed.gradient_norm(g).tolist()[0] - want) <= 140 * U32 * want


def test_more_tensors_than_a_launch_takes_and_none_gradients():
    sizes = [7 + i % 300 for i in range(300)]
    params, grads = tensors(sizes, F32), tensors(sizes, F32, seed=4)
    a, b = lm.AdamW([p.clone() for p in params]), lm.AdamW([p.clone() for p in params])
    a.step(grads, **HP)
    for i in range(300):                                   # one tensor at a time gives the same bits
        b.t = 0
        b.step([g if j == i else None for j, g in enumerate(grads)], **HP)
    for x, y in zip(a.params, b.params):
        assert torch.equal(x, y)
    assert torch.equal(a.moments["exp_avg_sq"], b.moments["exp_avg_sq"])


def decode(code, scale, second):
    """The format of include/jorge_lm.h, in 64 bits."""
    c, k = code.astype(np.int64), scale.astype(np.int64).repeat(lm.BLOCK) - 127
    mag, bias = (c, 15) if second else (c & 127, 7)
    e, man = mag >> 4, mag & 15
    y = np.where(e > 0, np.ldexp(1 + man / 16, e - bias), np.ldexp(man / 16, 1 - bias))
    return np.ldexp(y * (1 if second else np.where(c > 127, -1, 1)), k)


def random32(index, seed, t):
    m32 = np.uint64(0xFFFFFFFF)
    with np.errstate(over="ignore"):
        h = (index & m32) * np.uint64(0x9E3779B1) + np.uint64(seed * 0x85157AF5 + t * 0x2C9277B5)
        h &= m32
        h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x7C2E1B35)) & m32
        h = ((h ^ (h >> np.uint64(15))) * np.uint64(0x46D8C6A9)) & m32
        return (h ^ (h >> np.uint64(16))).astype(np.int64)


def test_every_code_reads_as_its_value():
    opt = lm.AdamW(tensors([512 * 256], F32), bits=8)
    for second, name in ((False, "exp_avg"), (True, "exp_avg_sq")):
        code = torch.arange(256, dtype=torch.uint8).repeat(512)
        scale = torch.arange(512).remainder(253).add(1).to(torch.uint8)
        opt.moments[name].copy_(code)
        opt.moments[name + "_scale"].copy_(scale)
        want = decode(code.numpy(), scale.numpy(), second)
        got = opt.moment_values()[int(second)].cpu().numpy()
        assert np.array_equal(got.astype(np.float64), want)
    zero = lm.AdamW(tensors([600], F32), bits=8)
    assert all(torch.count_nonzero(x) == 0 for x in zero.moment_values())


def check_rounding(x, code, scale, rnd, second, what):
    """Codes of 64-bit values x: the block's scale is the least that holds its largest, each value is one of x's
    two neighbours, and the upper one where the random bits say so (x in 32 bits may differ in its last places)."""
    x = np.where(np.abs(x) < 1e-42, 0.0, x)
    top = np.abs(x).reshape(-1, lm.BLOCK).max(1)
    k = scale.astype(np.int64) - 127
    assert np.all(top <= 31 / 16 * np.ldexp(1.0, k) * (1 + 1e-6)), what
    assert np.all((top > 31 / 16 * np.ldexp(1.0, k - 1) * (1 - 1e-6)) | (scale == 1)), what
    y = np.ldexp(np.abs(x), -k.repeat(lm.BLOCK))
    low = -14 if second else -6
    e = np.maximum(np.frexp(y)[1] - 1, low)
    part = np.ldexp(y, 4 - e)
    got = np.abs(np.ldexp(decode(code, scale, second), -k.repeat(lm.BLOCK)))
    steps = np.ldexp(got, 4 - e) - np.floor(part)
    if second:
        smallest = (steps == 1) & (np.floor(part) == 0) & (x > 0)      # never rounded to zero
    else:
        smallest = np.zeros_like(steps, dtype=bool)
        assert np.array_equal(np.sign(decode(code, scale, second))[got > 0], np.sign(x)[got > 0])
    frac = (part - np.floor(part)) * 65536
    clear = np.abs(np.floor(frac) + rnd - 65535.5) > 2
    clear &= (frac > 1) & (frac < 65535)
    up = np.floor(frac) + rnd >= 65536
    assert np.all((steps == up) | ~clear | smallest), what
    assert np.all((steps >= -1e-9) & (steps <= 1 + 1e-9) | ~clear), what
    assert not np.any(x) or clear[x != 0].mean() > 0.5, what       # the check reaches most values


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [1.0, 1e-12, 1e8])
def test_steps_in_8_bits(dtype, scale):
    sizes = [1000, 256, 5, 4099, 777]
    params = tensors(sizes, dtype)
    opt = lm.AdamW(params, bits=8, seed=11)
    for t in range(1, 4):
        grads = tensors(sizes, dtype, seed=t, scale=scale)
        grads[1].zero_()
        grads[3][:3000] *= 2.0 ** -9                       # a block's small elements: subnormal codes
        p, g = flat(opt, params), flat(opt, grads)
        m, v = (x.double().cpu() for x in opt.moment_values())
        opt.step(grads, **HP)
        p1, m1, v1, ms, vs, ps = formula(p, g, m, v, t, **HP)
        for i, (q, b) in enumerate(zip(params, opt.blocks)):
            s = slice(b * lm.BLOCK, b * lm.BLOCK + q.numel())
            within(q, p1[s], ps[s], 24, f"p{i}")
        rnd = random32(np.arange(len(p), dtype=np.uint64), 11, t)
        codes = {k: x.cpu().numpy() for k, x in opt.moments.items()}
        check_rounding(m1.numpy(), codes["exp_avg"], codes["exp_avg_scale"], rnd & 0xFFFF, False, f"m {t}")
        check_rounding(v1.numpy(), codes["exp_avg_sq"], codes["exp_avg_sq_scale"], rnd >> 16, True, f"v {t}")


def test_8_bit_rounding_is_even_handed():
    """A slow average follows its input in the mean: after many steps the 8-bit moments add up to the 32-bit ones."""
    n = 1 << 16
    g = tensors([n], F32, seed=3)
    a, b = lm.AdamW(tensors([n], F32)), lm.AdamW(tensors([n], F32), bits=8)
    for _ in range(300):
        for o in (a, b):
            o.step(g, lr=0.0, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0)
    for x, y in zip(a.moment_values(), b.moment_values()):
        # Independent errors of at most an eighth of a value each, its smallest codes apart.
        assert abs((y.double().sum() - x.double().sum()).item()) <= 5 * 0.125 * x.double().norm().item()
        assert (y - x).double().norm() <= 0.3 * x.double().norm()


def test_written_moments_are_rounded_to_nearest():
    opt = lm.AdamW(tensors([2048], F32), bits=8)
    m, v = tensors([2048], F32, seed=5)[0], tensors([2048], F32, seed=6)[0].square()
    m[256:512] = 0
    opt.set_moment_values(m, v)
    for got, want in zip(opt.moment_values(), (m, v)):
        top = want.abs().view(-1, 256).amax(1).repeat_interleave(256)
        # Half a step of four mantissa bits, or of the smallest normal code.
        assert bool(((got - want).abs() <= want.abs() / 32 + top * 2.0 ** -11).all())
    again = lm.AdamW(opt.params, bits=8, moments=opt.moments)
    assert torch.equal(again.moment_values()[0], opt.moment_values()[0])
    kept = [x.clone() for x in opt.moment_values()]
    opt.set_moment_values(*kept)                              # what a code stands for keeps its code
    assert all(torch.equal(x, y) for x, y in zip(kept, opt.moment_values()))


def test_nan_and_infinity_stay_in_their_elements():
    for bits in (32, 8):
        params, grads = tensors([600], F32), tensors([600], F32, seed=1)
        clean = lm.AdamW([params[0].clone()], bits=bits)
        clean.step([grads[0].clone()], **HP)
        grads[0][10], grads[0][300] = float("nan"), float("inf")
        opt = lm.AdamW(params, bits=bits)
        opt.step(grads, **HP)
        bad = torch.zeros(600, dtype=torch.bool, device="cuda")
        bad[[10, 300]] = True
        assert bool(torch.isnan(params[0][bad]).all()) and torch.equal(params[0][~bad], clean.params[0][~bad])


def test_views_at_odd_places_and_transposed_gradients():
    hold, ghold = tensors([5000], F32)[0], tensors([5000], F32, seed=1)[0]
    cut = lambda h: [h[1:400], h[401:1500], h[1503:4999]]  # noqa: E731
    copies = [p.clone() for p in cut(hold)]
    a, b = lm.AdamW(cut(hold), bits=8), lm.AdamW(copies, bits=8)
    edge = hold[[0, 400, 1500, 4999]].clone()
    a.step(cut(ghold), **HP)
    b.step([g.clone() for g in cut(ghold)], **HP)
    for x, y in zip(a.params, b.params):
        assert torch.equal(x, y)
    assert torch.equal(edge, hold[[0, 400, 1500, 4999]])
    p = tensors([24], F32)[0].view(4, 6)
    g = tensors([24], F32, seed=2)[0].view(6, 4).t()
    c, d = lm.AdamW([p.clone()]), lm.AdamW([p.clone()])
    c.step([g], **HP)
    d.step([g.contiguous()], **HP)
    assert torch.equal(c.params[0], d.params[0])


@pytest.mark.parametrize("bits", [32, 8])
def test_state_round_trip_resumes_bitwise(bits):
    params = tensors(SIZES, F32)
    opt = lm.AdamW(params, bits=bits, seed=3)
    opt.step(tensors(SIZES, F32, seed=1), **HP)
    buf = io.BytesIO()
    torch.save(opt.state_dict(), buf)
    buf.seek(0)
    twin = lm.AdamW([p.clone() for p in params], bits=bits)
    twin.load_state_dict(torch.load(buf, weights_only=True))
    for o in (opt, twin):
        o.step(tensors(SIZES, F32, seed=2), **HP)
    for x, y in zip(opt.params, twin.params):
        assert torch.equal(x, y)


def test_optimizer_groups_clip_together_and_resume():
    from paper_2310_12298_amd.optim import AdamWOptimizer

    def make():
        torch.manual_seed(0)
        return torch.nn.Sequential(torch.nn.Linear(40, 30), torch.nn.LayerNorm(30), torch.nn.Linear(30, 7)).cuda()

    def groups(m):
        vec = [p for p in m.parameters() if p.dim() < 2]
        return [{"params": [p for p in m.parameters() if p.dim() >= 2]},
                {"params": vec, "weight_decay": 0.0, "lr": 2e-3}]

    def backward(m, t):
        g = torch.Generator(device="cuda").manual_seed(t)
        for p in m.parameters():
            p.grad = torch.randn(p.shape, generator=g, device="cuda")

    a, b = make(), make()
    opt = AdamWOptimizer(groups(a), lr=1e-3, max_norm=1.0, bits=8, seed=5)
    ref = torch.optim.AdamW(groups(b), lr=1e-3, weight_decay=0.01, foreach=True)
    for t in range(1, 3):
        backward(a, t)
        backward(b, t)
        opt.step()
        norm = torch.nn.utils.clip_grad_norm_(b.parameters(), 1.0)
        assert abs(opt.norm - norm) <= 1e-5 * norm
        if t == 1:                                            # moments that have not been rounded yet
            ref.step()
            for x, y in zip(a.parameters(), b.parameters()):
                assert torch.allclose(x, y, rtol=1e-5, atol=1e-6)
    buf = io.BytesIO()
    torch.save(opt.state_dict(), buf)
    buf.seek(0)
    c = make()
    c.load_state_dict(a.state_dict())
    twin = AdamWOptimizer(groups(c), lr=1e-3, max_norm=1.0, bits=8)
    twin.load_state_dict(torch.load(buf, weights_only=True))
    for m, o in ((a, opt), (c, twin)):
        backward(m, 9)
        o.step()
    for x, y in zip(a.parameters(), c.parameters()):
        assert torch.equal(x, y)
    with pytest.raises(ValueError):
        AdamWOptimizer([torch.zeros(3)])


def test_a_parameter_that_moved_is_refused():
    p = torch.nn.Parameter(tensors([64], F32)[0].view(8, 8))
    opt = lm.AdamW([p])
    p.grad = torch.ones_like(p)
    opt.step()
    p.data = p.data.t()                                       # the moments are in the old order
    with pytest.raises(ValueError, match="has changed"):
        opt.step([torch.ones_like(p)])
    p.data = p.data.cpu()
    with pytest.raises(ValueError):
        opt.step([None])


def test_refusals():
    p = tensors([10, 20], F32)
    opt = lm.AdamW(p)
    g = [x.clone() for x in p]
    for bad in (lambda: lm.AdamW([x.cpu() for x in p]), lambda: lm.AdamW(p, bits=16), lambda: lm.AdamW([p[0][::2]]),
                lambda: lm.AdamW([x.half() for x in p]), lambda: opt.step(g[:1]), lambda: opt.step([g[0], g[1][:19]]),
                lambda: opt.step([g[0], g[1].bfloat16()]), lambda: lm.AdamW(p, moments={"exp_avg": p[0]}),
                lambda: lm.AdamW(p, bits=8).load_state_dict(opt.state_dict())):
        with pytest.raises(ValueError):
            bad()
    before = [x.clone() for x in p]
    for kw in (dict(lr=-1.0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=float("nan")),
               dict(weight_decay=float("inf")), dict(max_norm=-1.0)):
        with pytest.raises(lm.JorgeError):
            opt.step(g, **kw)
    assert opt.t == 0 and all(torch.equal(x, y) for x, y in zip(before, p))
    assert UNIT[F32] == U32
