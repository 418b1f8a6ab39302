"""The limits and workspaces of include/jorge_lm.h at their edges, without a GPU."""
import ctypes
import os
import re

import pytest

torch = pytest.importorskip("torch")

from paper_2310_12298_amd import lm  # noqa: E402
from test_lm_abi_host import A, HEADER, I64, INVALID, P, UNSUPPORTED, lib, refused  # noqa: E402, F401


def defined(name):
    value = re.search(rf"#define {name}\s+(\(1 << \d+\)|\d+)", open(HEADER).read()).group(1)
    a = re.match(r"\(1 << (\d+)\)", value)
    return 1 << int(a.group(1)) if a else int(value)


def test_row_strides_of_the_loss_end_where_the_header_says(lib):  # noqa: F811
    assert lm.LOSS_MAX_STRIDE == defined("JORGE_LOSS_MAX_STRIDE")
    n = I64()
    for ldh, ldw in ((8, lm.LOSS_MAX_STRIDE + 1), (lm.LOSS_MAX_STRIDE + 1, 8)):
        s = lm.LossShape(4, 8, 5, ldh, ldw, 1, 0, -100, 0.0)
        refused(lib, lib.jorge_cross_entropy_workspace(ctypes.byref(s), 0, ctypes.byref(n)), UNSUPPORTED, "MAX_STRIDE")
    s = lm.LossShape(4, 8, 5, lm.LOSS_MAX_STRIDE, lm.LOSS_MAX_STRIDE, 1, 0, -100, 0.0)
    assert lib.jorge_cross_entropy_workspace(ctypes.byref(s), 1, ctypes.byref(n)) == 0


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("tokens", [1, 63, 64, 700, 8192])
def test_the_loss_of_few_tokens_copies_no_whole_weight(lib, tokens, dtype):  # noqa: F811
    def size(vocab, back, cols=4096):
        s, n = lm.LossShape(tokens, cols, vocab, cols, cols, dtype, 0, -100, 0.0), I64()
        assert lib.jorge_cross_entropy_workspace(ctypes.byref(s), back, ctypes.byref(n)) == 0
        return n.value
    terms = 1 if dtype else 3
    for cols in (4096, 16384):
        # Twice 1 GiB of weight's copies; dz both ways round, 2^26 elements (fp32: half as many, of three terms);
        # hidden's two copies; the sums of its gradient, and two products' slices: 512 tiles of 256 x 256 floats each.
        most = 2 * 2 ** 30 + 2 * 2 * 2 ** 26 * (1 if dtype else 1.5) + 2 * 2 * terms * (tokens + 64) * cols
        most += 4 * tokens * cols + 2 * 512 * 256 * 256 * 4
        assert size(1 << 22, 1, cols) < most
        # Pieces of equal length are at least half as long as they may be.
        assert size(1 << 22, 1, cols) < 2 * size(1 << 18, 1, cols)


NO_GPU = pytest.mark.skipif(torch.cuda.is_available(), reason="accepted calls would follow made-up addresses")
HIP_ERROR = -3                                        # JORGE_ERR_HIP: of a launch, where there is no GPU


@NO_GPU
def test_8_bit_moments_are_read_and_written_at_any_size(lib):  # noqa: F811
    blocks = (1 << 23) + 300                          # 2^31 elements and more
    ms = lm.AdamWMoments(P(A), P(A), P(A), P(A), blocks, 8, 0)
    for second in (0, 1):
        for dtype in (0, 1):
            assert lib.jorge_adamw_read(ctypes.byref(ms), second, 0, blocks, P(A), dtype, None) == HIP_ERROR
        assert lib.jorge_adamw_write(ctypes.byref(ms), second, 0, blocks, P(A), None) == HIP_ERROR


@NO_GPU
@pytest.mark.parametrize("count", [0, 5, defined("JORGE_EMBED_MAX_TOKENS")])
@pytest.mark.parametrize("dtype", [0, 1])
def test_the_largest_table_is_not_refused_after_its_tokens_are_sorted(lib, count, dtype):  # noqa: F811
    vocab, cols = defined("JORGE_EMBED_MAX_VOCAB"), defined("JORGE_EMBED_MAX_COLS")
    n = I64()
    assert lib.jorge_embedding_workspace(count, vocab, cols, ctypes.byref(n)) == 0
    assert lib.jorge_embedding_backward(P(A), cols, P(A), count, dtype, vocab, cols, 1.0, -1, P(A), cols, P(A), n.value,
                                        None) == HIP_ERROR


def test_a_gradient_too_large_for_the_norm_has_no_workspace(lib):  # noqa: F811
    n = I64()
    for numel, want in ((1 << 38, 0), ((1 << 38) + 1, UNSUPPORTED), ((1 << 63) - 1, UNSUPPORTED), (-1, INVALID)):
        ts = (lm.AdamWTensor * 1)(lm.AdamWTensor(0, A, numel, 0, 0, 0))
        assert lib.jorge_gradient_norm_workspace(ts, 1, ctypes.byref(n)) == want
    assert n.value > (1 << 38) // (1 << 14) * 8       # of the one that was taken
