"""The C ABI of include/jorge_lm.h without a GPU: every entry point is exported and bound, the header compiles as
C11 and as C++, refusals come before any HIP call and say why, and the workspaces' sizes are sane."""
import ctypes
import os
import re
import subprocess

import pytest

pytest.importorskip("torch")

from paper_2310_12298_amd import jorge as J  # noqa: E402
from paper_2310_12298_amd import lm  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "jorge_lm.h")
INVALID, UNSUPPORTED = -1, -4
P, I64 = ctypes.c_void_p, ctypes.c_int64
A = 1 << 20                                            # an address that no refused call follows


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(J.LIB_PATH):
        from paper_2310_12298_amd.build import build_library
        build_library()
    return lm.load_operators()


def refused(lib, status, want, why):
    assert status == want and why in lib.jorge_lm_last_error().decode(), (status, lib.jorge_lm_last_error())


def test_every_declared_symbol_is_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(jorge_[a-z_]+)\s*\(", text))
    assert names == set(lm._SIGNATURES) and all(hasattr(lib, n) for n in names)


@pytest.mark.parametrize("compiler", [["gcc", "-std=c11"], ["g++", "-std=c++17", "-x", "c++"]])
def test_header_stands_alone(tmp_path, compiler):
    src = tmp_path / "h.c"
    src.write_text('#include "jorge_lm.h"\nint main(void) { return sizeof(jorge_adamw_tensor) == 40 ? 0 : 1; }\n')
    subprocess.run([*compiler, "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(tmp_path / "h")], check=True)
    assert subprocess.run([str(tmp_path / "h")]).returncode == 0
    assert ctypes.sizeof(lm.AdamWTensor) == 40


def test_layer_norm_refusals(lib):
    def forward(x=A, ldx=8, dtype=0, w=A, b=A, pd=0, y=A, ldy=8, mean=A, rstd=A, rows=4, cols=8, eps=1e-5):
        return lib.jorge_layernorm_forward(P(x), ldx, dtype, P(w), P(b), pd, P(y), ldy, P(mean), P(rstd), rows, cols,
                                           eps, None)
    for kw, why in ((dict(dtype=2), "type"), (dict(pd=-1), "type"), (dict(rows=-1), "rows"), (dict(cols=0), "cols"),
                    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
                    (dict(ldx=7), "stride"), (dict(ldy=7), "stride"), (dict(x=None), "x and y"),
                    (dict(mean=None), "mean"),
                    (dict(x=A + 2), "aligned"), (dict(w=A + 1), "aligned")):
        refused(lib, forward(**kw), INVALID, why)
    refused(lib, forward(cols=16385, ldx=16385, ldy=16385), UNSUPPORTED, "MAX_COLS")
    assert forward(rows=0, x=None, y=None) == 0        # nothing to do

    def backward(dy=A, x=A, mean=A, w=A, dx=A, dw=A, rows=4, cols=8, ld=8, ws=A, n=1 << 20):
        return lib.jorge_layernorm_backward(P(dy), ld, P(x), ld, 0, P(mean), P(A), P(w), 0, P(dx), ld, P(dw), P(A),
                                            rows, cols, P(ws), n, None)
    for kw, why in ((dict(dy=None), "needed"), (dict(mean=None), "needed"), (dict(ws=None), "workspace"),
                    (dict(ws=A + 16), "workspace"), (dict(n=100), "too small"), (dict(ld=7), "stride")):
        refused(lib, backward(**kw), INVALID, why)


def test_embedding_refusals(lib):
    def forward(tok=A, n=4, table=A, ldt=8, dtype=1, vocab=5, cols=8, scale=1.0, out=A, ldo=8):
        return lib.jorge_embedding_forward(P(tok), n, P(table), ldt, dtype, vocab, cols, scale, P(out), ldo, None)
    for kw, why in ((dict(n=-1), "count"), (dict(vocab=0), "vocab"), (dict(cols=0), "cols"), (dict(dtype=3), "type"),
                    (dict(scale=float("inf")), "scale"), (dict(ldt=7), "stride"), (dict(tok=None), "needed"),
                    (dict(tok=A + 4), "aligned"), (dict(out=A + 1), "aligned")):
        refused(lib, forward(**kw), INVALID, why)
    refused(lib, forward(n=(1 << 24) + 1), UNSUPPORTED, "MAX_TOKENS")
    refused(lib, forward(vocab=(1 << 24) + 1), UNSUPPORTED, "MAX_VOCAB")
    refused(lib, forward(cols=32769, ldt=32769, ldo=32769), UNSUPPORTED, "MAX_COLS")

    def backward(d=A, tok=A, n=4, dt=A, ws=A, size=1 << 20):
        return lib.jorge_embedding_backward(P(d), 8, P(tok), n, 0, 5, 8, 1.0, -1, P(dt), 8, P(ws), size, None)
    for kw, why in ((dict(d=None), "needed"), (dict(dt=None), "needed"), (dict(ws=None), "workspace"),
                    (dict(size=8), "too small")):
        refused(lib, backward(**kw), INVALID, why)


def test_cross_entropy_refusals(lib):
    def shape(tokens=4, cols=8, vocab=5, ldh=8, ldw=8, dtype=1, ignore=-100, smoothing=0.0):
        return lm.LossShape(tokens, cols, vocab, ldh, ldw, dtype, 0, ignore, smoothing)

    def forward(h=A, w=A, t=A, loss=A, total=A, ws=A, size=1 << 30, **kw):
        return lib.jorge_cross_entropy_forward(ctypes.byref(shape(**kw)), P(h), P(w), P(t), P(loss), P(A), P(total),
                                               P(ws), size, None)
    for kw, why in ((dict(tokens=-1), "tokens"), (dict(cols=0), "cols"), (dict(vocab=0), "vocab"),
                    (dict(dtype=4), "type"), (dict(ldh=7), "stride"), (dict(ldw=7), "stride"),
                    (dict(smoothing=1.01), "smoothing"),
                    (dict(smoothing=float("nan")), "smoothing"), (dict(h=None), "needed"), (dict(t=A + 4), "aligned"),
                    (dict(w=A + 1), "aligned"), (dict(total=None), "total"), (dict(ws=A + 8), "workspace"),
                    (dict(size=64), "too small")):
        refused(lib, forward(**kw), INVALID, why)
    for kw, why in ((dict(tokens=(1 << 21) + 1), "TOKENS"), (dict(vocab=(1 << 22) + 1), "VOCAB"),
                    (dict(cols=32769, ldh=32769, ldw=32769), "COLS"), (dict(ldw=(1 << 22) + 1), "stride")):
        refused(lib, forward(**kw), UNSUPPORTED, why)

    def backward(kind=0, grad=A, lse=A, dh=A, ws=A, size=1 << 30, **kw):
        return lib.jorge_cross_entropy_backward(ctypes.byref(shape(**kw)), P(grad), kind, P(A), P(A), P(A), P(lse),
                                                P(A), P(dh), P(A), P(ws), size, None)
    for kw, why in ((dict(kind=3), "kind"), (dict(kind=-1), "kind"), (dict(grad=None), "needed"),
                    (dict(lse=None), "needed"),
                    (dict(dh=A + 1), "aligned"), (dict(ws=None), "workspace"), (dict(size=64), "too small")):
        refused(lib, backward(**kw), INVALID, why)
    n = I64()
    assert lib.jorge_cross_entropy_workspace(None, 0, ctypes.byref(n)) == INVALID
    sizes = {}
    for tokens in (0, 1, 63, 8192, 1 << 21):
        for vocab in (1, 50001, 1 << 22):
            for dtype in (0, 1):
                for back in (0, 1):
                    s = shape(tokens=tokens, vocab=vocab, cols=2048, ldh=2048, ldw=2048, dtype=dtype)
                    assert lib.jorge_cross_entropy_workspace(ctypes.byref(s), back, ctypes.byref(n)) == 0
                    assert n.value % 256 == 0 and (n.value > 0) == (tokens > 0)
                    sizes[tokens, vocab, dtype, back] = n.value
    # The logits are not kept: a large vocabulary takes no more than a piece of it does.
    assert sizes[8192, 1 << 22, 1, 1] < 1.2 * sizes[8192, 50001, 1, 1] < 8192 * 50001 * 4


def test_adamw_refusals(lib):
    def step(numels=(300, 10), blocks=(0, 2), held=3, bits=32, dtype=0, t=1, ptr=A, scale=A, m=A, **kw):
        ts = (lm.AdamWTensor * len(numels))(*[lm.AdamWTensor(ptr, A, n, b, dtype, 0) for n, b in zip(numels, blocks)])
        ms = lm.AdamWMoments(P(m), P(A), P(scale), P(scale), held, bits, 0)
        h = {**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, wd=0.0), **kw}
        return lib.jorge_adamw_step(ts, len(numels), ctypes.byref(ms), t, h["lr"], h["beta1"], h["beta2"], h["eps"],
                                    h["wd"], None, None)
    for kw, why in ((dict(blocks=(0, 1)), "overlap"), (dict(held=2), "within"), (dict(blocks=(2, 0)), "ascend"),
                    (dict(bits=16), "bits"), (dict(dtype=7), "type"), (dict(t=0), "t >= 1"), (dict(ptr=0), "null"),
                    (dict(ptr=A + 2), "aligned"), (dict(bits=8, scale=None), "scales"), (dict(m=None), "buffers"),
                    (dict(m=A + 4), "16 bytes"), (dict(lr=-1.0), "lr"), (dict(eps=float("nan")), "eps"),
                    (dict(beta1=1.0), "betas"), (dict(beta2=float("nan")), "betas"), (dict(numels=(-1, 4)), "numel"),
                    (dict(held=-1), "blocks"), (dict(blocks=(-1, 2)), "blocks")):
        refused(lib, step(**kw), INVALID, why)
    assert lib.jorge_adamw_step(None, 1, None, 1, 0.1, 0.9, 0.9, 0.1, 0.0, None, None) == INVALID
    ms = lm.AdamWMoments(P(A), P(A), P(A), P(A), 3, 8, 0)
    for args, why in (((0, 0, 4, P(A), 0), "outside"), ((0, 3, 1, P(A), 0), "outside"), ((2, 0, 1, P(A), 0), "second"),
                      ((0, 0, 1, None, 0), "buffer"), ((1, 0, 1, P(A), 5), "type")):
        refused(lib, lib.jorge_adamw_read(ctypes.byref(ms), *args, None), INVALID, why)
    refused(lib, lib.jorge_adamw_write(ctypes.byref(ms), 0, -1, 1, P(A), None), INVALID, "outside")
    ts = (lm.AdamWTensor * 1)(lm.AdamWTensor(0, A, 5, 0, 0, 0))
    for args, why in (((-1.0, P(A), P(A), 256), "max_norm"), ((0.0, None, P(A), 256), "out"),
                      ((0.0, P(A), None, 256), "workspace"), ((0.0, P(A), P(A), 8), "too small")):
        refused(lib, lib.jorge_gradient_norm(ts, 1, *args, None), INVALID, why)


def test_workspaces_are_multiples_of_256(lib):
    n = I64()
    for rows, cols in ((0, 1), (1, 1), (5, 16384), (1 << 20, 4096)):
        assert lib.jorge_layernorm_workspace(rows, cols, ctypes.byref(n)) == 0 and n.value % 256 == 0
        assert n.value <= 768 * 2 * cols * 4 + 256
    for count, vocab, cols in ((0, 1, 1), (1, 5, 3), (16384, 50000, 2048), (1 << 24, 1 << 24, 8)):
        assert lib.jorge_embedding_workspace(count, vocab, cols, ctypes.byref(n)) == 0 and n.value % 256 == 0
        assert n.value >= 8 * count
    assert lib.jorge_layernorm_workspace(1, 1, None) == INVALID
    assert lib.jorge_embedding_workspace(1, 1, 0, ctypes.byref(n)) == INVALID


def test_operators_need_a_gpu_tensor():
    import torch
    for call in (lambda: lm.layer_norm_forward(torch.ones(2, 3)),
                 lambda: lm.embedding_forward(torch.zeros(2).long(), torch.ones(2, 3)),
                 lambda: lm.AdamW([torch.ones(3)])):
        with pytest.raises(ValueError, match="CUDA"):
            call()
