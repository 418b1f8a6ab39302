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
