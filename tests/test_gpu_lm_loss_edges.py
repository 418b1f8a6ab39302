"""Cross entropy over a vocabulary on the GPU where it is called in less usual ways, against the formula in 64 bits or
against the usual call's bits."""
import pytest

torch = pytest.importorskip("torch")

from paper_2310_12298_amd import lm  # noqa: E402
from test_gpu_lm_loss import BF16, F32, check, inputs, plain  # noqa: E402

pytestmark = pytest.mark.gpu


def one(value=1.0):
    return torch.tensor(value, device="cuda")


def relative(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("dtype,of_targets,of_others", [
    # A rounding to eight bits errs evenly within 2^-8 of the power of two at or below a value: 2^-8 / sqrt(3) of it at
    # most. Rows of words without a target have one such error in each term of their sums, independently, and one more.
    (BF16, 2 ** -8 / 3 ** 0.5, 2 ** -8 * (2 / 3) ** 0.5),
    # Three-term splits: the sums' own roundings, independent: sqrt(6 512 / 32) of a logit of size two, and
    # sqrt(6 8192 / 32) of dhidden's sums, 1.2e-6 and 2.3e-6; twice that together.
    (F32, 5e-6, 5e-6)])
def test_whom_the_rounding_of_dz_costs(dtype, of_targets, of_others):
    h, w, t = inputs(1024, 512, 8192, dtype, ignored=0.0)
    t = (t % 500)                                            # few words are targets
    loss, lse, total = lm.cross_entropy_forward(h, w, t)
    dh, dw = lm.cross_entropy_backward(one(), h, w, t, lse, total)
    want = plain(h, w, t, 0.0, -100, lambda live: torch.full_like(live, 1 / 1024, dtype=torch.float64))
    hit = torch.zeros(8192, dtype=torch.bool, device="cuda")
    hit[t] = True
    assert relative(dh, want["dh"]) < of_targets
    assert relative(dw[hit], want["dw"][hit]) < of_targets
    assert relative(dw[~hit], want["dw"][~hit]) < of_others


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,v", [(128, 4096, 32000), (162, 1984, 35280), (70, 200, 900)])
def test_weight_that_cannot_be_read_in_place(n, d, v, dtype):
    """It goes in pieces of the vocabulary, whose tiles may differ from those of weight in place: both hold against
    64 bits, each gives the same bits again, and so does the backward pass of both."""
    h, w, t = inputs(n, d, v, dtype)
    lse, total = lm.cross_entropy_forward(h, w, t)[1:]
    grads = lm.cross_entropy_backward(one(), h, w, t, lse, total)
    for start, pad in ((1, 0), (0, 8), (3, 1)):
        hold = torch.full((v * (d + pad) + start,), float("nan"), dtype=dtype, device="cuda")
        x = hold[start:].view(v, d + pad)[:, :d]
        x.copy_(w)
        check(h, x, t)
        assert all(torch.equal(a, b) for a, b in zip(*(lm.cross_entropy_forward(h, x, t) for _ in range(2))))
        got = lm.cross_entropy_backward(one(), h, x, t, lse, total)
        assert all(torch.equal(a, b) for a, b in zip(got, grads))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_last_tokens_of_long_sequences(dtype):
    """hidden[:, -1]: rows further apart than the C call takes, both passes and through autograd."""
    n, length, d, v = 3, 9000, 512, 700
    h, w, t = inputs(n, d, v, dtype, ignored=0.0)
    whole = torch.zeros(n, length, d, dtype=dtype, device="cuda")
    whole[:, -1] = h
    last = whole[:, -1]
    assert last.stride(0) > lm.LOSS_MAX_STRIDE
    base = lm.cross_entropy_forward(h, w, t)
    assert all(torch.equal(a, b) for a, b in zip(lm.cross_entropy_forward(last, w, t), base))
    want = lm.cross_entropy_backward(one(), h, w, t, *base[1:])
    assert all(torch.equal(a, b) for a, b in zip(lm.cross_entropy_backward(one(), last, w, t, *base[1:]), want))
    whole.requires_grad_()
    lm.linear_cross_entropy(whole[:, -1], w, t).backward()
    assert torch.equal(whole.grad[:, -1], want[0]) and torch.count_nonzero(whole.grad[:, :-1]) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_narrow_slices_take_no_more_than_twice_their_size(dtype):
    h, w, t = inputs(64, 128, 300, dtype)
    wide_h, wide_w = (torch.full((m.shape[0], 5000), float("nan"), dtype=dtype, device="cuda") for m in (h, w))
    wide_h[:, 8:136], wide_w[:, 16:144] = h, w
    base = lm.cross_entropy_forward(h, w, t)
    got = lm.cross_entropy_backward(one(), wide_h[:, 8:136], wide_w[:, 16:144], t, *base[1:])
    for a, b in zip(got, lm.cross_entropy_backward(one(), h, w, t, *base[1:])):
        assert torch.equal(a, b) and a.untyped_storage().nbytes() <= 2 * b.numel() * b.element_size()


@pytest.mark.parametrize("n,d,v,dtype", [(5, 4096, 60000, F32), (66, 4096, 60001, F32), (3, 16384, 40000, BF16)])
def test_few_tokens_over_several_pieces(n, d, v, dtype):
    """Pieces that weight's copies bound, not dz."""
    check(*inputs(n, d, v, dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,v", [(90, 72, 300), (40, 64, 9000), (4000, 64, 20000)])
def test_rows_without_a_target_get_no_gradient_whatever_comes_in(n, d, v, dtype):
    """The upstream gradient of a step whose loss overflowed, and weights that have: a masked row's gradient stays 0.
    Sizes with one range of K, with several, and with several pieces of the vocabulary."""
    h, w, t = inputs(n, d, v, dtype)
    t[0] = -100
    masked = t < 0
    lse, total = lm.cross_entropy_forward(h, w, t)[1:]
    for reduction in ("mean", "sum", "none"):
        for value in (float("inf"), float("nan")):
            grad = torch.full((n,), value, device="cuda") if reduction == "none" else one(value)
            dh, dw = lm.cross_entropy_backward(grad, h, w, t, lse, total, reduction)
            assert torch.count_nonzero(dh[masked]) == 0 and not bool(torch.isfinite(dh[~masked]).any())
            none = torch.full_like(t, -100)
            total0 = lm.cross_entropy_forward(h, w, none)[2]
            for x in lm.cross_entropy_backward(grad, h, w, none, lse, total0, reduction):
                assert torch.count_nonzero(x) == 0
    bad = w.clone()
    bad[3, 5] = float("inf")
    lse, total = lm.cross_entropy_forward(h, bad, t)[1:]
    dh = lm.cross_entropy_backward(one(), h, bad, t, lse, total)[0]
    assert torch.count_nonzero(dh[masked]) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,v,start", [(150, 96, 700, 0), (150, 96, 700, 1), (4000, 64, 20000, 0),
                                         (5, 4096, 60000, 0)])
def test_one_gradient_alone_has_the_same_bits(n, d, v, start, dtype):
    h, w, t = inputs(n, d, v, dtype)
    hold = torch.zeros(v * d + start, dtype=dtype, device="cuda")
    x = hold[start:].view(v, d)
    x.copy_(w)
    lse, total = lm.cross_entropy_forward(h, x, t)[1:]
    dh, dw = lm.cross_entropy_backward(one(), h, x, t, lse, total)
    a = lm.cross_entropy_backward(one(), h, x, t, lse, total, need_weight=False)
    b = lm.cross_entropy_backward(one(), h, x, t, lse, total, need_hidden=False)
    assert a[1] is None and b[0] is None and torch.equal(a[0], dh) and torch.equal(b[1], dw)
    assert lm.cross_entropy_backward(one(), h, x, t, lse, total, need_hidden=False, need_weight=False) == (None, None)


def test_autograd_forms_only_the_gradients_that_are_asked_for():
    h, w, t = inputs(30, 40, 90, F32)
    want = []
    for a, b in ((True, True), (True, False), (False, True)):
        x, y = h.clone().requires_grad_(a), w.clone().requires_grad_(b)
        lm.linear_cross_entropy(x, y, t).backward()
        want = want or [x.grad, y.grad]
        for g, ref, asked in ((x.grad, want[0], a), (y.grad, want[1], b)):
            assert torch.equal(g, ref) if asked else g is None


def test_an_infinite_weight_in_fp32_takes_its_word_from_rows_where_the_logit_is_minus_infinity():
    """As a weight so large that the word's probability is 0 there does: to the bit."""
    h, w, t = inputs(90, 72, 300, F32)
    t[t == 3] = 4
    rows = h[:, 5] < 0
    lost = []
    for big in (1e30, 3.4e38, float("inf")):
        w[3, 5] = big
        lost.append([x[rows] for x in lm.cross_entropy_forward(h, w, t, label_smoothing=0.0)[:2]])
    assert bool(torch.isfinite(lost[0][1]).all()) and int(rows.sum()) > 20
    for other in lost[1:]:
        assert all(torch.equal(a, b) for a, b in zip(lost[0], other))
