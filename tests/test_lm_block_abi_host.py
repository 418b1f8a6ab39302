"""The linear, gated linear and attention calls of include/jorge_lm.h without a GPU: refusals come before any HIP call
and say why, limits are the header's, workspaces are sane, and the largest accepted sizes reach a launch."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2310_12298_amd import lm  # noqa: E402
from test_lm_abi_host import A, I64, INVALID, P, ROOT, UNSUPPORTED, lib, refused  # noqa: E402, F401
from test_lm_limits_host import HIP_ERROR, NO_GPU, defined  # noqa: E402

BIG = 1 << 40


def test_structures_are_the_headers(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include "jorge_lm.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu", '
                   'sizeof(jorge_linear_shape), sizeof(jorge_heads), sizeof(jorge_attention_shape)); return 0; }\n')
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "h")],
                   check=True)
    sizes = subprocess.run([str(tmp_path / "h")], capture_output=True, text=True).stdout.split()
    assert [int(n) for n in sizes] == [ctypes.sizeof(t) for t in (lm.LinearShape, lm.Heads, lm.AttentionShape)]


def test_limits_are_the_headers():
    assert lm.LINEAR_MAX_STRIDE == defined("JORGE_LINEAR_MAX_STRIDE")
    assert lm.LINEAR_FEW_TOKENS == defined("JORGE_LINEAR_FEW_TOKENS")
    assert lm.ATTENTION_MAX_STRIDE == defined("JORGE_ATTENTION_MAX_STRIDE")
    for name, value in (("RELU", 1), ("GELU", 2), ("SILU", 3), ("SIGMOID", 4), ("NONE", 0)):
        assert defined("JORGE_ACT_" + name) == value == lm.ACTIVATIONS[name.lower()]


def linear_shape(tokens=100, cols=8, outs=12, ldx=None, ldw=None, ldu=None, ldy=None, ldr=None, dtype=1, bias_dtype=0,
                 act=0):
    return lm.LinearShape(tokens, cols, outs, ldx or cols, ldw or cols, ldu or cols, ldy or outs, ldr or outs, dtype,
                          bias_dtype, act, 0)


SHAPES = ((dict(tokens=-1), INVALID, "tokens"), (dict(cols=0, ldx=1, ldw=1, ldu=1), INVALID, "cols"),
          (dict(outs=0, ldy=1), INVALID, "outs"), (dict(dtype=2), INVALID, "type"), (dict(act=5), INVALID, "activation"),
          (dict(act=-1), INVALID, "activation"), (dict(ldx=7), INVALID, "stride"), (dict(ldw=7), INVALID, "stride"),
          (dict(ldy=11), INVALID, "stride"), (dict(tokens=(1 << 21) + 1), UNSUPPORTED, "MAX_TOKENS"),
          (dict(cols=32769), UNSUPPORTED, "MAX_COLS"), (dict(outs=(1 << 18) + 1), UNSUPPORTED, "MAX_OUTS"),
          (dict(tokens=1 << 21, cols=32768), UNSUPPORTED, "2^34"), (dict(ldw=(1 << 22) + 1), UNSUPPORTED, "MAX_STRIDE"))


def test_linear_refusals(lib):  # noqa: F811
    def forward(x=A, w=A, b=A, r=A, y=A, ws=A, size=BIG, **kw):
        return lib.jorge_linear_forward(ctypes.byref(linear_shape(**kw)), P(x), P(w), P(b), P(r), P(y), P(ws), size, None)
    for kw, status, why in SHAPES + ((dict(bias_dtype=7), INVALID, "bias"), (dict(x=None), INVALID, "needed"),
                                     (dict(y=None), INVALID, "needed"), (dict(w=A + 1), INVALID, "aligned"),
                                     (dict(r=A + 1), INVALID, "aligned"), (dict(b=A + 2), INVALID, "aligned"),
                                     (dict(ldr=11), INVALID, "stride"), (dict(ws=None), INVALID, "workspace"),
                                     (dict(ws=A + 8), INVALID, "workspace"), (dict(size=64), INVALID, "too small")):
        refused(lib, forward(**kw), status, why)
    assert lib.jorge_linear_forward(None, *[P(A)] * 6, BIG, None) == INVALID
    assert forward(tokens=0, x=None, y=None, ws=None) == 0

    def backward(dy=A, x=A, w=A, b=A, dx=A, dw=A, db=A, lddx=8, lddw=8, ws=A, size=BIG, **kw):
        return lib.jorge_linear_backward(ctypes.byref(linear_shape(**kw)), P(dy), P(x), P(w), P(b), P(dx), lddx, P(dw),
                                         lddw, P(db), P(ws), size, None)
    for kw, status, why in SHAPES + ((dict(dy=None), INVALID, "needed"), (dict(x=None), INVALID, "needed"),
                                     (dict(dx=A + 1), INVALID, "aligned"), (dict(db=A + 2), INVALID, "aligned"),
                                     (dict(lddx=7), INVALID, "stride"), (dict(lddw=7), INVALID, "stride"),
                                     (dict(ws=None), INVALID, "workspace"), (dict(size=64), INVALID, "too small")):
        refused(lib, backward(**kw), status, why)
    assert backward(dx=None, dw=None, db=None) == 0      # nothing is asked for


def test_gated_linear_refusals(lib):  # noqa: F811
    def forward(x=A, g=A, u=A, y=A, ws=A, size=BIG, **kw):
        return lib.jorge_gated_linear_forward(ctypes.byref(linear_shape(**kw)), P(x), P(g), P(u), P(y), P(ws), size, None)
    more = ((dict(ldu=7), INVALID, "stride"), (dict(u=None), INVALID, "needed"), (dict(u=A + 1), INVALID, "aligned"),
            (dict(ws=None), INVALID, "workspace"), (dict(size=64), INVALID, "too small"))
    for kw, status, why in SHAPES + more:
        refused(lib, forward(**kw), status, why)

    def backward(dy=A, g=A, u=A, dx=A, dg=A, du=A, lddw=8, ws=A, size=BIG, **kw):
        return lib.jorge_gated_linear_backward(ctypes.byref(linear_shape(**kw)), P(dy), P(A), P(g), P(u), P(dx), 8,
                                               P(dg), P(du), lddw, P(ws), size, None)
    for kw, status, why in SHAPES + more + ((dict(dg=None), INVALID, "together"), (dict(du=None), INVALID, "together"),
                                            (dict(lddw=7), INVALID, "stride"), (dict(dy=None), INVALID, "needed")):
        refused(lib, backward(**kw), status, why)
    assert backward(dx=None, dg=None, du=None) == 0


def test_linear_workspaces(lib):  # noqa: F811
    n = I64()

    def size(gated, back, **kw):
        assert lib.jorge_linear_workspace(ctypes.byref(linear_shape(**kw)), gated, back, ctypes.byref(n)) == 0
        assert n.value % 256 == 0
        return n.value
    assert lib.jorge_linear_workspace(None, 0, 0, ctypes.byref(n)) == INVALID
    assert lib.jorge_linear_workspace(ctypes.byref(linear_shape()), 0, 0, None) == INVALID
    for gated in (0, 1):
        for dtype in (0, 1):
            few = dict(cols=2048, outs=8192, dtype=dtype, act=3)
            assert size(gated, 0, tokens=0, **few) == size(gated, 1, tokens=0, **few) == 0
            assert size(gated, 0, tokens=1, **few) == size(gated, 0, tokens=lm.LINEAR_FEW_TOKENS, **few) == 0
            assert size(gated, 0, tokens=lm.LINEAR_FEW_TOKENS + 1, **few) > 0 < size(gated, 1, tokens=1, **few)
    # dz, and copies of what may have to be copied, of two bytes an element; nothing grows with tokens * tokens.
    most = 2 * (8192 * 2 * 8192 + 8192 * 2048 + 2 * 8192 * 2048) + (1 << 20)
    assert size(1, 1, tokens=8192, cols=2048, outs=8192, act=3) < most


@pytest.mark.parametrize("gated,act", [(0, 0), (0, 3), (1, 3)])
@pytest.mark.parametrize("tokens,cols,outs", [(8192, 8192, 8192), (1515, 7854, 230), (1950000, 17, 8200),
                                              (130, 4001, 70), (4096, 2048, 1 << 17)])
def test_ranges_of_fp32_sums_take_at_most_a_gibibyte(lib, tokens, cols, outs, gated, act):  # noqa: F811
    """Beside the copies of three bfloat16 terms an element, of rows padded to 64, and dbias's parts."""
    n = I64()
    s = linear_shape(tokens=tokens, cols=cols, outs=outs, dtype=0, act=act)
    assert lib.jorge_linear_workspace(ctypes.byref(s), gated, 1, ctypes.byref(n)) == 0
    mats, (kd, kf, kn) = 1 + gated, (-(-v // 64) * 64 for v in (cols, outs, tokens))
    again = tokens * kd + mats * outs * kd if gated or act else 0       # for z, formed again
    terms = again + cols * kn + cols * mats * kf + tokens * mats * kf + mats * outs * kn
    parts = 0 if gated else (tokens // (32 if act else 128) + 2) * outs
    assert n.value <= 6 * terms + 4 * parts + (1 << 30) + (1 << 13)


def call_workspace(lib, dy=None, x=A, w=A, u=None, wanted=0, **kw):  # noqa: F811
    n = I64()
    assert lib.jorge_linear_call_workspace(ctypes.byref(linear_shape(**kw)), P(dy), P(x), P(w), P(u), wanted,
                                           ctypes.byref(n)) == 0
    return n.value


def test_a_calls_workspace_has_room_for_what_the_call_uses(lib):  # noqa: F811
    for name in ("DX", "DWEIGHT", "DBIAS"):
        assert getattr(lm, "LINEAR_" + name) == defined("JORGE_LINEAR_" + name)
    n = I64()
    assert lib.jorge_linear_call_workspace(None, None, P(A), P(A), None, 0, ctypes.byref(n)) == INVALID
    assert lib.jorge_linear_call_workspace(ctypes.byref(linear_shape()), None, P(A), P(A), None, 0, None) == INVALID
    for kw, status, why in SHAPES:
        refused(lib, lib.jorge_linear_call_workspace(ctypes.byref(linear_shape(**kw)), None, P(A), P(A), None, 0,
                                                     ctypes.byref(n)), status, why)
    plain = dict(tokens=8192, cols=8192, outs=2048)
    # bfloat16 operands that can be read as they lie need nothing without an activation, and dz with one.
    assert call_workspace(lib, **plain) == call_workspace(lib, A, wanted=3, **plain) == 0
    assert call_workspace(lib, A, wanted=3, act=3, **plain) == 2 * 8192 * 2048
    assert call_workspace(lib, A, u=A, wanted=3, act=3, **plain) == 2 * 8192 * 2 * 2048
    # One that cannot be is copied.
    assert call_workspace(lib, x=A + 8, **plain) == 2 * 8192 * 8192
    assert call_workspace(lib, w=A + 8, **plain) == 2 * 2048 * 8192
    assert call_workspace(lib, u=A + 8, **plain) == 2 * 2 * 2048 * 8192
    assert call_workspace(lib, A + 8, wanted=3, **plain) == 2 * 8192 * 2048
    assert call_workspace(lib, ldx=8193, **plain) == 2 * 8192 * 8192
    # Gradients that are not asked for take none, and in fp32 none of their copies.
    assert call_workspace(lib, A, **plain) == call_workspace(lib, tokens=0) == call_workspace(lib, A, wanted=7, tokens=0) == 0
    plain["dtype"] = 0
    every = call_workspace(lib, A, wanted=3, act=3, **plain)
    for wanted in (1, 2, 4):
        assert 0 < call_workspace(lib, A, wanted=wanted, act=3, **plain) < every
    dw = 6 * 8192 * (8192 + 2048)                                     # x and dz across their rows
    assert every - call_workspace(lib, A, wanted=1, act=3, **plain) >= dw


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("tokens,cols,outs", [(1, 96, 40), (64, 64, 64), (65, 64, 192), (300, 200, 130), (2048, 4096, 64),
                                              (515, 512, 1000), (8192, 2048, 8192), (182, 5702, 6326)])
def test_a_calls_workspace_is_no_more_than_any_calls(lib, tokens, cols, outs, dtype):  # noqa: F811
    n = I64()
    for act in (0, 3):
        kw = dict(tokens=tokens, cols=cols, outs=outs, dtype=dtype, act=act)
        s = linear_shape(**kw)
        for u in (None, A, A + 4):
            most = []
            for back in (0, 1):
                assert lib.jorge_linear_workspace(ctypes.byref(s), int(u is not None), back, ctypes.byref(n)) == 0
                most.append(n.value)
            for at in (A, A + 4):
                assert call_workspace(lib, x=at, w=at, u=u, **kw) <= most[0]
                for wanted in range(8):
                    assert call_workspace(lib, at, A, at, u, wanted, **kw) <= most[1]


@NO_GPU
@pytest.mark.parametrize("dtype", [0, 1])
def test_a_calls_workspace_is_what_the_call_takes(lib, dtype):  # noqa: F811
    """With it the launches are reached, with less the call is refused."""
    for tokens, cols, outs, act in ((515, 512, 1024, 0), (300, 200, 130, 3), (130, 4001, 70, 3), (2048, 4096, 64, 2)):
        kw = dict(tokens=tokens, cols=cols, outs=outs, dtype=dtype, act=act)
        s = linear_shape(**kw)

        def tried(need, call):
            if need:
                refused(lib, call(need - 256), INVALID, "too small")
            assert call(need) == HIP_ERROR
        for at in (A, A + 4):
            tried(call_workspace(lib, x=at, **kw), lambda size: lib.jorge_linear_forward(
                ctypes.byref(s), P(at), P(A), P(A), P(A), P(A), P(A), size, None))
            tried(call_workspace(lib, x=at, u=A, **kw), lambda size: lib.jorge_gated_linear_forward(
                ctypes.byref(s), P(at), P(A), P(A), P(A), P(A), size, None))
            for wanted in range(1, 8):
                dx, dw, db = (P(A) if wanted & bit else None for bit in (1, 2, 4))
                tried(call_workspace(lib, A, at, wanted=wanted, **kw), lambda size: lib.jorge_linear_backward(
                    ctypes.byref(s), P(A), P(at), P(A), P(A), dx, cols, dw, cols, db, P(A), size, None))
                if wanted < 4:
                    tried(call_workspace(lib, A, at, u=A, wanted=wanted, **kw),
                          lambda size: lib.jorge_gated_linear_backward(ctypes.byref(s), P(A), P(at), P(A), P(A), dx, cols,
                                                                       dw, dw, cols, P(A), size, None))


def attention_shape(batch=2, q=5, kv=9, heads=4, kv_heads=2, dim=16, dtype=1, scale=0.25, causal=0, window=0, ql=None,
                    kl=None, qp=A, kp=A, vp=A, token=256, head=16):
    at = (token * 16, token, head)
    return lm.AttentionShape(batch, q, kv, heads, kv_heads, dim, dtype, scale, causal, 0, window, ql, kl, qp, *at, kp,
                             *at, vp, *at)


def heads(p=A, batch=4096, token=256, head=16):
    return ctypes.byref(lm.Heads(p, batch, token, head))


ATTENTION = ((dict(batch=-1), INVALID, "batch"), (dict(q=-1), INVALID, "tokens"), (dict(dtype=2), INVALID, "type"),
             (dict(kv_heads=3), INVALID, "multiple"), (dict(heads=0), INVALID, "multiple"),
             (dict(kv_heads=0), INVALID, "multiple"), (dict(dim=0), INVALID, "dim"), (dict(scale=0.0), INVALID, "scale"),
             (dict(scale=-1.0), INVALID, "scale"), (dict(scale=float("nan")), INVALID, "scale"),
             (dict(scale=float("inf")), INVALID, "scale"), (dict(causal=2), INVALID, "causal"),
             (dict(window=-1, causal=1), INVALID, "window"), (dict(window=3), INVALID, "causal"),
             (dict(dim=129), UNSUPPORTED, "MAX_DIM"), (dict(q=(1 << 22) + 1), UNSUPPORTED, "MAX_TOKENS"),
             (dict(kv=(1 << 22) + 1), UNSUPPORTED, "MAX_TOKENS"),
             (dict(batch=1 << 10, heads=64, q=1 << 11), UNSUPPORTED, "MAX_ROWS"))
INPUTS = ((dict(qp=None), INVALID, "q is needed"), (dict(kp=None), INVALID, "k is needed"),
          (dict(vp=None), INVALID, "v is needed"), (dict(qp=A + 1), INVALID, "aligned"),
          (dict(kl=A + 4), INVALID, "aligned"), (dict(token=(1 << 22) + 1), UNSUPPORTED, "MAX_STRIDE"),
          (dict(token=-1), INVALID, "negative"))


def test_attention_refusals(lib):  # noqa: F811
    n = I64()

    def forward(out=heads(), lse=A, ws=A, size=BIG, **kw):
        return lib.jorge_attention_forward(ctypes.byref(attention_shape(**kw)), out, P(lse), P(ws), size, None)
    for kw, status, why in ATTENTION + INPUTS + (
            (dict(out=None), INVALID, "needed"), (dict(lse=None), INVALID, "needed"), (dict(lse=A + 2), INVALID, "aligned"),
            (dict(out=heads(None)), INVALID, "out is needed"), (dict(out=heads(A + 1)), INVALID, "aligned"),
            (dict(dim=5, ws=None), INVALID, "workspace"), (dict(dim=5, ws=A + 8), INVALID, "workspace"),
            (dict(dim=5, size=64), INVALID, "too small")):
        refused(lib, forward(**kw), status, why)
    for kw, status, why in ATTENTION:
        refused(lib, lib.jorge_attention_workspace(ctypes.byref(attention_shape(**kw)), None, ctypes.byref(n)), status, why)
    assert lib.jorge_attention_workspace(None, None, ctypes.byref(n)) == INVALID
    assert lib.jorge_attention_workspace(ctypes.byref(attention_shape()), None, None) == INVALID
    assert forward(batch=0, out=None, lse=None) == 0 and forward(q=0, out=None, lse=None) == 0

    def backward(dout=heads(), out=heads(), lse=A, dq=heads(), dk=heads(), dv=heads(), ws=A, size=BIG, **kw):
        return lib.jorge_attention_backward(ctypes.byref(attention_shape(**kw)), dout, out, P(lse), dq, dk, dv, P(ws),
                                            size, None)
    for kw, status, why in ATTENTION + INPUTS + (
            (dict(dout=None), INVALID, "needed"), (dict(out=None), INVALID, "needed"), (dict(lse=None), INVALID, "needed"),
            (dict(dq=heads(A + 1)), INVALID, "aligned"), (dict(dv=heads(A, token=-5)), INVALID, "negative"),
            (dict(ws=None), INVALID, "workspace"), (dict(size=64), INVALID, "too small")):
        refused(lib, backward(**kw), status, why)
    assert backward(dq=None, dk=None, dv=None) == 0 and backward(batch=0) == 0


def test_attention_workspaces(lib):  # noqa: F811
    n = I64()

    def size(dout=None, **kw):
        assert lib.jorge_attention_workspace(ctypes.byref(attention_shape(**kw)), dout, ctypes.byref(n)) == 0
        assert n.value % 256 == 0
        return n.value
    # A batch that fills the card and can be read as it lies needs nothing forward, two numbers a row backward.
    train = dict(batch=4, q=4096, kv=4096, heads=16, kv_heads=16, dim=128)
    assert size(**train) == 0 and size(heads(), **train) == 2 * 4 * 4 * 16 * 4096
    # One that cannot be is copied: q, k and v, and the gradient.
    odd = dict(train, dim=127)
    assert size(**odd) == 3 * 2 * 4 * 4096 * 16 * 128 and size(heads(), **odd) > 4 * 2 * 4 * 4096 * 16 * 128
    # A long cache under one token is read in place, and its ranges' results are small.
    assert 0 < size(batch=1, q=1, kv=1 << 20, heads=32, kv_heads=8, dim=128) < 1 << 22
    assert size(batch=0) == 0


def test_rows_of_q_and_of_k_are_limited_each_by_its_own_heads(lib):  # noqa: F811
    """A step of generation for many sequences has few rows of q, with all heads, and many of k, with kv_heads."""
    most = defined("JORGE_ATTENTION_MAX_ROWS")
    n = I64()

    def status(dout=None, **kw):
        return lib.jorge_attention_workspace(ctypes.byref(attention_shape(**kw)), dout, ctypes.byref(n))
    for batch, kv in ((64, 32768), (16, 131072)):
        step = dict(batch=batch, q=1, kv=kv, heads=64, kv_heads=8, dim=128)
        assert batch * 64 * kv > most >= batch * 8 * kv
        assert status(**step) == 0 and status(heads(), **step) == 0
    assert status(batch=1 << 10, q=1, kv=most >> 13, heads=64, kv_heads=8) == 0
    refused(lib, status(batch=1 << 10, q=1, kv=(most >> 13) + 1, heads=64, kv_heads=8), UNSUPPORTED, "kv_heads")
    assert status(batch=1 << 10, q=most >> 16, kv=1, heads=64, kv_heads=8) == 0
    refused(lib, status(batch=1 << 10, q=(most >> 16) + 1, kv=1, heads=64, kv_heads=8), UNSUPPORTED, "q_tokens")


@NO_GPU
@pytest.mark.parametrize("dtype", [0, 1])
def test_the_largest_sizes_are_launched(lib, dtype):  # noqa: F811
    n = I64()
    for kw in (dict(tokens=1 << 21, cols=8192, outs=8192), dict(tokens=1 << 16, cols=32768, outs=1 << 18),
               dict(tokens=1, cols=32768, outs=1 << 18)):
        s = linear_shape(**kw, dtype=dtype, act=3, ldw=lm.LINEAR_MAX_STRIDE)
        for gated in (0, 1):
            assert lib.jorge_linear_workspace(ctypes.byref(s), gated, 0, ctypes.byref(n)) == 0
            args = (P(A), P(A), P(A)) if gated else (P(A), P(A), P(A), P(A))
            call = lib.jorge_gated_linear_forward if gated else lib.jorge_linear_forward
            assert call(ctypes.byref(s), *args, P(A), P(A), n.value, None) == HIP_ERROR
            assert lib.jorge_linear_workspace(ctypes.byref(s), gated, 1, ctypes.byref(n)) == 0
            c = s.cols
            if gated:
                assert lib.jorge_gated_linear_backward(ctypes.byref(s), P(A), P(A), P(A), P(A), P(A), c, P(A), P(A), c,
                                                       P(A), n.value, None) == HIP_ERROR
            else:
                assert lib.jorge_linear_backward(ctypes.byref(s), P(A), P(A), P(A), P(A), P(A), c, P(A), c, P(A), P(A),
                                                 n.value, None) == HIP_ERROR
    for kw in (dict(batch=1, q=1 << 22, kv=1 << 22, heads=16, kv_heads=4, dim=128),
               dict(batch=1 << 20, q=1, kv=16, heads=4, kv_heads=4, dim=5)):
        s = attention_shape(**kw, dtype=dtype, token=lm.ATTENTION_MAX_STRIDE)
        assert lib.jorge_attention_workspace(ctypes.byref(s), None, ctypes.byref(n)) == 0
        assert lib.jorge_attention_forward(ctypes.byref(s), heads(), P(A), P(A), n.value, None) == HIP_ERROR
        assert lib.jorge_attention_workspace(ctypes.byref(s), heads(), ctypes.byref(n)) == 0
        assert lib.jorge_attention_backward(ctypes.byref(s), heads(), heads(), P(A), heads(), heads(), heads(), P(A),
                                            n.value, None) == HIP_ERROR
