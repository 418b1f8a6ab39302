"""Embedding lookup and its gradient on the GPU against indexing and sums in 64 bits.

Roundings of a gradient's sum: at most 32 rows (4096 positions and more: 64 and so on) by the wave,
then its chunks' sums by eighths, eight at a time: below 32 + chunks / 8 + 16. One more for the scale.
"""
import pytest

torch = pytest.importorskip("torch")

from lm_check import slope, within  # noqa: E402
from paper_2310_12298_amd import lm  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def plain_grad(dout, tokens, vocab, scale, padding=None):
    d, t = dout.double().cpu(), tokens.cpu()
    ok = (t >= 0) & (t < vocab)
    if padding is not None:
        ok &= t != padding
    out, size = (torch.zeros(vocab, dout.shape[1], dtype=torch.float64) for _ in range(2))
    out.index_add_(0, t[ok], d[ok] * scale)
    size.index_add_(0, t[ok], d[ok].abs() * abs(scale))
    return out, size


def check_grad(tokens, vocab, cols, dtype, scale=1.5, padding=None, seed=0):
    g = torch.Generator().manual_seed(seed)
    dout = torch.randn(len(tokens), cols, generator=g).to(dtype).cuda()
    got = lm.embedding_backward(dout, tokens.cuda(), vocab, scale, padding)
    assert got.dtype == dtype and got.shape == (vocab, cols)
    want, size = plain_grad(dout, tokens, vocab, scale, padding)
    within(got, want, size, 64 + len(tokens) / 256, "dtable")
    assert torch.equal(got, lm.embedding_backward(dout, tokens.cuda(), vocab, scale, padding))   # the same bits again


def some_tokens(kind, n, vocab):
    g = torch.Generator().manual_seed(n + vocab)
    if kind == "uniform":
        return torch.randint(0, vocab, (n,), generator=g)
    if kind == "one":
        return torch.full((n,), vocab - 1)
    if kind == "half":
        t = torch.randint(0, vocab, (n,), generator=g)
        t[torch.rand(n, generator=g) < 0.5] = vocab // 2
        return t
    if kind == "sorted":
        return (torch.arange(n) * vocab // n).clamp(max=vocab - 1)
    t = torch.randint(-3, vocab + 3, (n,), generator=g)      # "strays": some outside the table
    t[0] = 1 << 40
    t[-1] = -(1 << 40)
    return t


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["uniform", "one", "half", "sorted", "strays"])
@pytest.mark.parametrize("n,vocab,cols", [(1, 1, 1), (2, 5, 3), (31, 7, 64), (32, 40, 65), (33, 257, 8),
                                          (1000, 100, 130), (1025, 65536, 5), (4097, 300, 516), (16384, 999, 24),
                                          (16385, 4000, 12)])
def test_gradient(kind, n, vocab, cols, dtype):
    check_grad(some_tokens(kind, n, vocab), vocab, cols, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 2, 4, 5, 9, 16, 23, 33, 64, 127, 128, 129, 256, 257])
def test_rows_without_tokens(cols, dtype):
    """A wave looks for the tokens of 64 rows: vocabularies that end inside them, and rows of every width."""
    for n in (3, 1500, 2048, 2049):
        check_grad(some_tokens("uniform", n, 200 if n < 100 else 5003), 200 if n < 100 else 5003, cols, dtype)


@pytest.mark.parametrize("kind", ["uniform", "half", "one"])
def test_gradient_over_several_tiles_and_merges(kind):
    check_grad(some_tokens(kind, 16384 * 3 + 77, 70000), 70000, 4, F32)
    check_grad(some_tokens(kind, 16384 * 8 + 1, 300), 300, 8, F32)        # a second merge, of a run of one
    check_grad(some_tokens(kind, 16384 * 17 + 5, 1 << 17), 1 << 17, 2, F32)


def test_gradient_keeps_the_order_of_positions():
    """A run's sum is left to right within its chunk: sums that cancel exactly in that order alone."""
    vocab, n = 5, 20
    tokens = torch.full((n,), 3)
    dout = torch.zeros(n, 1)
    dout[0], dout[1], dout[2] = 2.0 ** 30, 1.0, -(2.0 ** 30)              # (2^30 + 1) - 2^30 = 0 in 32 bits
    got = lm.embedding_backward(dout.cuda(), tokens.cuda(), vocab)
    assert got[3, 0].item() == 0.0
    got = lm.embedding_backward(dout[[0, 2, 1] + list(range(3, n))].cuda(), tokens.cuda(), vocab)
    assert got[3, 0].item() == 1.0


def test_padding_gets_no_gradient_and_strides_do_not_matter():
    tokens = some_tokens("half", 700, 50)
    check_grad(tokens, 50, 33, F32, padding=25)
    g = torch.Generator().manual_seed(1)
    hold = torch.randn(700 * 41 + 3, generator=g).cuda()
    dout = hold[3:].view(700, 41)[:, :33]
    got = lm.embedding_backward(dout, tokens.cuda(), 50, 2.0)
    assert torch.equal(got, lm.embedding_backward(dout.contiguous(), tokens.cuda(), 50, 2.0))


def test_no_tokens():
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert torch.count_nonzero(lm.embedding_backward(torch.empty(0, 9, device="cuda"), none, 6)) == 0
    out = lm.embedding_forward(none, torch.ones(3, 9, device="cuda"))
    assert out.shape == (0, 9)


def test_nan_and_infinity_stay_in_their_row():
    tokens = torch.tensor([1, 2, 1, 4, 2])
    dout = torch.ones(5, 10)
    dout[2, 3], dout[3, 9] = float("nan"), float("-inf")
    got = lm.embedding_backward(dout.cuda(), tokens.cuda(), 6).cpu()
    assert bool(torch.isnan(got[1, 3])) and got[4, 9] == float("-inf") and torch.isfinite(got).sum() == 58


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [1, 3, 8, 17, 64, 100, 511, 1024, 2050, 9000])
def test_forward(cols, dtype):
    g = torch.Generator().manual_seed(cols)
    table = torch.randn(37, cols, generator=g).to(dtype).cuda()
    tokens = torch.randint(-1, 38, (3, 50), generator=g).cuda()
    out = lm.embedding_forward(tokens, table, scale=3.7)
    t = tokens.cpu()
    want = table.double().cpu()[t.clamp(0, 36)] * 3.7 * ((t >= 0) & (t < 37))[..., None]
    assert out.shape == (3, 50, cols)
    within(out, want, want.abs(), 2, "out")                               # the scale's rounding, the product's
    hold = torch.zeros(37, cols + 5, dtype=dtype, device="cuda")
    hold[:, 2:cols + 2] = table
    assert torch.equal(lm.embedding_forward(tokens, hold[:, 2:cols + 2], scale=3.7), out)
    assert torch.equal(lm.embedding_forward(tokens.int(), table, scale=3.7), out)


def test_autograd_and_differences():
    g = torch.Generator().manual_seed(3)
    table = torch.randn(20, 6, generator=g).cuda().requires_grad_()
    tokens = torch.randint(0, 20, (4, 9), generator=g).cuda()
    dy = torch.randn(4, 9, 6, generator=g).cuda()
    lm.embedding(tokens, table, scale=0.5, padding=7).backward(dy)
    v = torch.randn(20, 6, generator=g, dtype=torch.float64)
    keep = (tokens != 7).cpu()[..., None]
    f = lambda t: (0.5 * t[tokens.cpu()] * dy.double().cpu() * keep).sum()  # noqa: E731
    want = slope(f, table.detach().double().cpu(), v, 1e-3)
    got = (table.grad.double().cpu() * v).sum()
    assert abs(got - want) <= 1e-6 * table.grad.double().norm().cpu() * v.norm()


def test_refusals():
    table, tokens = torch.ones(5, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    dout = torch.ones(4, 8, device="cuda")
    for bad in (lambda: lm.embedding_forward(tokens.float(), table), lambda: lm.embedding_forward(tokens, table.half()),
                lambda: lm.embedding_forward(tokens.cpu(), table), lambda: lm.embedding_forward(tokens, table[0]),
                lambda: lm.embedding_backward(dout[:3], tokens, 5),
                lambda: lm.embedding_backward(dout, tokens, 5, padding=5)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lm.embedding_forward(tokens, table, scale=float("nan")),
                lambda: lm.embedding_backward(dout, tokens, 0),
                lambda: lm.embedding_backward(dout, tokens, (1 << 24) + 1)):
        with pytest.raises(lm.JorgeError):
            bad()
