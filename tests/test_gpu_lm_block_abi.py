"""The C interface's own freedoms in linear layers and attention, which the Python functions make no use of: outputs in
rows wider than they are, whose gaps stay as they were, a result that takes its residual's place, gradients side by side
in one matrix. Where results go has no part in what they are: every one equals the plain call's bit for bit."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2310_12298_amd import lm  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
GAP = 777.0                                        # what the gaps hold (exact in both types)
SIZES = [(1, 96, 40), (17, 130, 65), (70, 64, 192), (300, 200, 130), (515, 512, 1000)]


def rand(g, *shape, d):
    return torch.randn(shape, generator=g).to(d).cuda()


def space(lib, call, *args):
    n = ctypes.c_int64(0)
    assert getattr(lib, call)(*args, ctypes.byref(n)) == 0
    return torch.empty(max(1, n.value), dtype=torch.uint8, device="cuda"), n.value


def stream():
    return torch.cuda.current_stream().cuda_stream


def shape_of(n, d, f, dtype, act, ldy, ldr):
    return lm.LinearShape(n, d, f, d, d, d, ldy, ldr, lm.DTYPES[dtype], lm.DTYPES[F32], lm.ACTIVATIONS[act], 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", SIZES)
def test_a_linear_layers_result_in_wider_rows_and_in_its_residuals_place(n, d, f, dtype):
    lib = lm.load_operators()
    g = torch.Generator().manual_seed(n + d + f)
    x, w, b = rand(g, n, d, d=dtype), rand(g, f, d, d=dtype), rand(g, f, d=F32)
    wide = torch.full((n, f + 3), GAP, dtype=dtype, device="cuda")
    residual = rand(g, n, f, d=dtype)
    for act in (None, "gelu"):
        shape = shape_of(n, d, f, dtype, act, f + 3, f + 3)
        ws, size = space(lib, "jorge_linear_workspace", ctypes.byref(shape), 0, 0)
        want = lm.linear_forward(x, w, b, act, residual)
        wide[:, :f] = residual
        assert lib.jorge_linear_forward(ctypes.byref(shape), x.data_ptr(), w.data_ptr(), b.data_ptr(), wide.data_ptr(),
                                        wide.data_ptr(), ws.data_ptr(), size, stream()) == 0
        assert torch.equal(wide[:, :f], want)
        assert bool((wide[:, f:] == GAP).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d,f", SIZES)
def test_gradients_of_linear_layers_in_wider_rows(n, d, f, dtype):
    lib = lm.load_operators()
    g = torch.Generator().manual_seed(n * d + f)
    x, w, u, dy = rand(g, n, d, d=dtype), rand(g, f, d, d=dtype), rand(g, f, d, d=dtype), rand(g, n, f, d=dtype)
    for act in (None, "silu"):
        shape = shape_of(n, d, f, dtype, act, f, f)
        dx = torch.full((n, d + 5), GAP, dtype=dtype, device="cuda")
        dw, du = (torch.full((f, d + 1), GAP, dtype=dtype, device="cuda") for _ in range(2))
        ws, size = space(lib, "jorge_linear_workspace", ctypes.byref(shape), 0, 1)
        assert lib.jorge_linear_backward(ctypes.byref(shape), dy.data_ptr(), x.data_ptr(), w.data_ptr(), None,
                                         dx.data_ptr(), d + 5, dw.data_ptr(), d + 1, None, ws.data_ptr(), size,
                                         stream()) == 0
        want = lm.linear_backward(dy, x, w, None, act)
        for got, to in ((dx, want[0]), (dw, want[1])):
            assert torch.equal(got[:, :d], to) and bool((got[:, d:] == GAP).all())
        ws, size = space(lib, "jorge_linear_workspace", ctypes.byref(shape), 1, 1)
        assert lib.jorge_gated_linear_backward(ctypes.byref(shape), dy.data_ptr(), x.data_ptr(), w.data_ptr(),
                                               u.data_ptr(), dx.data_ptr(), d + 5, dw.data_ptr(), du.data_ptr(), d + 1,
                                               ws.data_ptr(), size, stream()) == 0
        want = lm.gated_linear_backward(dy, x, w, u, act)
        for got, to in ((dx, want[0]), (dw, want[1]), (du, want[2])):
            assert torch.equal(got[:, :d], to) and bool((got[:, d:] == GAP).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,heads,kv_heads,dim", [(1, 4, 2, 64), (33, 3, 3, 20), (200, 4, 1, 80), (515, 2, 2, 128)])
def test_attentions_results_side_by_side_in_one_matrix(n, heads, kv_heads, dim, dtype):
    """o in wider rows; dq, dk and dv in the layout that one projection gives q, k and v: heads side by side."""
    lib = lm.load_operators()
    g = torch.Generator().manual_seed(n + dim)
    batch, all_heads = 2, heads + 2 * kv_heads
    qkv = rand(g, batch, n, all_heads, dim, d=dtype)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 2)
    dout = rand(g, batch, n, heads, dim, d=dtype)
    shape, _ = lm._attention_args(q, k, v, None, True, None, None, None)
    out = torch.full((batch, n, heads, dim + 8), GAP, dtype=dtype, device="cuda")
    lse = torch.empty((batch, heads, n), device="cuda")

    def heads_of(t):
        return lm.Heads(t.data_ptr(), *t.stride()[:3])

    ws, size = space(lib, "jorge_attention_workspace", ctypes.byref(shape), None)
    assert lib.jorge_attention_forward(ctypes.byref(shape), ctypes.byref(heads_of(out)), lse.data_ptr(), ws.data_ptr(),
                                       size, stream()) == 0
    want, want_lse = lm.attention_forward(q, k, v, causal=True)
    assert torch.equal(out[..., :dim], want) and torch.equal(lse, want_lse)
    assert bool((out[..., dim:] == GAP).all())
    grad = torch.full((batch, n, all_heads + 1, dim), GAP, dtype=dtype, device="cuda")
    hd = heads_of(dout)
    ws, size = space(lib, "jorge_attention_workspace", ctypes.byref(shape), ctypes.byref(hd))
    parts = grad.split([heads, kv_heads, kv_heads, 1], 2)
    assert lib.jorge_attention_backward(ctypes.byref(shape), ctypes.byref(hd), ctypes.byref(heads_of(out)),
                                        lse.data_ptr(), *[ctypes.byref(heads_of(t)) for t in parts[:3]], ws.data_ptr(),
                                        size, stream()) == 0
    for got, to in zip(parts, lm.attention_backward(dout, q, k, v, want, want_lse, causal=True)):
        assert torch.equal(got, to)
    assert bool((parts[3] == GAP).all())
