"""Operators of a language model's training step beside the Jorge step: layer norm, embedding,
cross entropy over a vocabulary, and AdamW with the global gradient norm.

ctypes binding of include/jorge_lm.h. layer_norm(), embedding() and linear_cross_entropy() are
differentiable; the *_forward and *_backward functions are the two passes by themselves; AdamW
steps a list of tensors. torch owns the memory (outputs and workspaces are torch tensors of the
current stream) and names the current HIP stream. Tensors are fp32 or bfloat16 CUDA tensors of the
current device; the last dimension has to be dense, rows may have a stride. There is no CPU
fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import warnings

import numpy as np
import torch

from .jorge import JORGE_OK, JorgeError, load_library

_P, _I32, _I64, _F64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
BLOCK = 256                                   # elements of an 8-bit moment that share a scale
DTYPES = {torch.float32: 0, torch.bfloat16: 1}
REDUCTIONS = {"none": 0, "sum": 1, "mean": 2}


class LossShape(ctypes.Structure):
    _fields_ = [("tokens", _I64), ("cols", _I64), ("vocab", _I64), ("ldh", _I64), ("ldw", _I64), ("dtype", _I32),
                ("reserved", _I32), ("ignore_index", _I64), ("label_smoothing", _F64)]


class AdamWTensor(ctypes.Structure):
    # Addresses as numbers, so that a numpy view of an array of these can set them by the column.
    _fields_ = [("param", ctypes.c_uint64), ("grad", ctypes.c_uint64), ("numel", _I64), ("block", _I64),
                ("dtype", _I32), ("reserved", _I32)]


class AdamWMoments(ctypes.Structure):
    _fields_ = [("exp_avg", _P), ("exp_avg_sq", _P), ("exp_avg_scale", _P), ("exp_avg_sq_scale", _P),
                ("blocks", _I64), ("bits", _I32), ("seed", ctypes.c_uint32)]


_PT, _PM, _PS = ctypes.POINTER(AdamWTensor), ctypes.POINTER(AdamWMoments), ctypes.POINTER(LossShape)
# name -> (restype, argtypes); mirrors include/jorge_lm.h
_SIGNATURES = {
    "jorge_lm_last_error": (ctypes.c_char_p, []),
    "jorge_layernorm_forward": (_I32, [_P, _I64, _I32, _P, _P, _I32, _P, _I64, _P, _P, _I64, _I64, _F64, _P]),
    "jorge_layernorm_workspace": (_I32, [_I64, _I64, ctypes.POINTER(_I64)]),
    "jorge_layernorm_backward": (_I32, [_P, _I64, _P, _I64, _I32, _P, _P, _P, _I32, _P, _I64, _P, _P, _I64, _I64, _P,
                                        _I64, _P]),
    "jorge_embedding_forward": (_I32, [_P, _I64, _P, _I64, _I32, _I64, _I64, _F64, _P, _I64, _P]),
    "jorge_embedding_workspace": (_I32, [_I64, _I64, _I64, ctypes.POINTER(_I64)]),
    "jorge_embedding_backward": (_I32, [_P, _I64, _P, _I64, _I32, _I64, _I64, _F64, _I64, _P, _I64, _P, _I64, _P]),
    "jorge_cross_entropy_workspace": (_I32, [_PS, _I32, ctypes.POINTER(_I64)]),
    "jorge_cross_entropy_forward": (_I32, [_PS, _P, _P, _P, _P, _P, _P, _P, _I64, _P]),
    "jorge_cross_entropy_backward": (_I32, [_PS, _P, _I32, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _P]),
    "jorge_gradient_norm_workspace": (_I32, [_PT, _I32, ctypes.POINTER(_I64)]),
    "jorge_gradient_norm": (_I32, [_PT, _I32, _F64, _P, _P, _I64, _P]),
    "jorge_adamw_step": (_I32, [_PT, _I32, _PM, _I64, _F64, _F64, _F64, _F64, _F64, _P, _P]),
    "jorge_adamw_read": (_I32, [_PM, _I32, _I64, _I64, _P, _I32, _P]),
    "jorge_adamw_write": (_I32, [_PM, _I32, _I64, _I64, _P, _P]),
}

_BOUND = None


def load_operators() -> ctypes.CDLL:
    """The library with the entry points of include/jorge_lm.h bound; raises if it is not built."""
    global _BOUND
    lib = load_library()
    if _BOUND is not lib:
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _BOUND = lib
    return lib


def _stream(t=None):
    """The current HIP stream of t's device as a number (torch's own shortcut: a Stream object takes 3 us to make)."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if t is None else t.get_device())


def _check(lib, status):
    if status != JORGE_OK:
        raise JorgeError(status, f"{lib.jorge_status_string(status).decode()} ({lib.jorge_lm_last_error().decode()})")


def _cuda(t, what, dtypes=DTYPES):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what}: a CUDA tensor is needed")
    if t.dtype not in dtypes:
        raise ValueError(f"{what}: unsupported type {t.dtype}")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what}: on device {t.get_device()}, not the current one")
    return t


def _matrix(t, what):
    """A matrix with dense rows that holds t's values, without a copy where t's layout allows it."""
    _cuda(t, what)
    dims = t.dim()
    if dims == 2:
        if t.is_contiguous():
            return t
        m = t
    elif dims == 0:
        raise ValueError(f"{what}: at least one dimension is needed")
    else:
        m = t.reshape(t.shape[:-1].numel(), t.shape[-1])
    if (m.shape[1] > 1 and m.stride(1) != 1) or (m.shape[0] > 1 and m.stride(0) < m.shape[1]):
        m = m.contiguous()
    return m


def _ld(m):
    """Row stride of a matrix; that of a single row does not matter."""
    return m.stride(0) if m.shape[0] > 1 else m.shape[1]


def _vector(t, n, what):
    _cuda(t, what)
    if tuple(t.shape) != (n,):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, not {(n,)}")
    return t.contiguous()


def _int64s(t, what):
    if isinstance(t, torch.Tensor) and t.dtype is torch.int64 and t.is_contiguous():
        return _cuda(t, what, (torch.int64,))
    if not isinstance(t, torch.Tensor) or t.dtype.is_floating_point or t.dtype.is_complex or t.dtype == torch.bool:
        raise ValueError(f"{what}: a tensor of whole numbers is needed")
    return _cuda(t.long().contiguous(), what, (torch.int64,))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


# ---------------------------------------------------------------- layer norm
def layer_norm_forward(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of layer norm over the last dimension; y has x's shape and type, mean and
    rstd are fp32, one per row. weight, bias: fp32 or bfloat16 vectors (one type), or None."""
    lib = load_operators()
    m = _matrix(x, "x")
    rows, cols = m.shape
    params = [_vector(p, cols, n) for p, n in ((weight, "weight"), (bias, "bias")) if p is not None]
    if len({p.dtype for p in params}) > 1:
        raise ValueError("weight and bias must have one type")
    w = params[0] if weight is not None else None
    b = params[-1] if bias is not None else None
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean = torch.empty(rows, dtype=torch.float32, device=x.device)
    rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(lib, lib.jorge_layernorm_forward(m.data_ptr(), _ld(m), DTYPES[x.dtype], _ptr(w), _ptr(b),
                                            DTYPES[params[0].dtype] if params else 0, y.data_ptr(), cols,
                                            mean.data_ptr(), rstd.data_ptr(), rows, cols, float(eps),
                                            _stream(x)))
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, affine=True):
    """(dx, dweight, dbias) from the gradient of y and what layer_norm_forward returned. dweight and
    dbias have weight's type (fp32 without one); affine=False leaves them out (None)."""
    lib = load_operators()
    m, d = _matrix(x, "x"), _matrix(dy, "dy")
    rows, cols = m.shape
    if tuple(dy.shape) != tuple(x.shape) or dy.dtype != x.dtype:
        raise ValueError("dy must have x's shape and type")
    for s, what in ((mean, "mean"), (rstd, "rstd")):
        if _cuda(s, what, (torch.float32,)).shape != (rows,) or not s.is_contiguous():
            raise ValueError(f"{what}: as layer_norm_forward returned it")
    w = None if weight is None else _vector(weight, cols, "weight")
    ptype = torch.float32 if w is None else w.dtype
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw = db = ws = None
    n = _I64(0)
    if affine:
        dw = torch.empty(cols, dtype=ptype, device=x.device)
        db = torch.empty(cols, dtype=ptype, device=x.device)
        _check(lib, lib.jorge_layernorm_workspace(rows, cols, ctypes.byref(n)))
        ws = _workspace(n.value)
    _check(lib, lib.jorge_layernorm_backward(d.data_ptr(), _ld(d), m.data_ptr(), _ld(m), DTYPES[x.dtype],
                                             mean.data_ptr(), rstd.data_ptr(), _ptr(w), DTYPES[ptype], dx.data_ptr(),
                                             cols, _ptr(dw), _ptr(db), rows, cols, _ptr(ws), n.value,
                                             _stream(x)))
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, mean, rstd, weight, bias)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, mean, rstd, weight, bias = ctx.saved_tensors
        need_w, need_b = ctx.needs_input_grad[1], ctx.needs_input_grad[2]
        dx, dw, db = layer_norm_backward(dy, x, mean, rstd, weight, affine=need_w or need_b)
        return dx, dw if need_w else None, db.to(bias.dtype) if need_b else None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Differentiable layer norm over the last dimension (see layer_norm_forward)."""
    return _LayerNorm.apply(x, weight, bias, eps)


# ---------------------------------------------------------------- embedding
def embedding_forward(tokens, table, scale=1.0):
    """scale * table[tokens], of table's type. A token outside the table gives a row of zeros."""
    lib = load_operators()
    t, tok = _matrix(table, "table"), _int64s(tokens, "tokens")
    if table.dim() != 2:
        raise ValueError("table: a matrix is needed")
    vocab, cols = t.shape
    out = torch.empty(tokens.shape + (cols,), dtype=t.dtype, device=t.device)
    _check(lib, lib.jorge_embedding_forward(tok.data_ptr(), tok.numel(), t.data_ptr(), _ld(t), DTYPES[t.dtype], vocab,
                                            cols, float(scale), out.data_ptr(), cols, _stream(t)))
    return out


def embedding_backward(dout, tokens, vocab, scale=1.0, padding=None):
    """The gradient of embedding_forward's table (vocab rows, dout's type). padding: a token whose row gets none."""
    lib = load_operators()
    d, tok = _matrix(dout, "dout"), _int64s(tokens, "tokens")
    if tuple(dout.shape[:-1]) != tuple(tokens.shape):
        raise ValueError(f"dout: shape {tuple(dout.shape)} for tokens of shape {tuple(tokens.shape)}")
    if padding is not None and not 0 <= int(padding) < int(vocab):
        raise ValueError("padding must be a row of the table")
    count, cols = d.shape
    n = _I64(0)
    _check(lib, lib.jorge_embedding_workspace(count, int(vocab), cols, ctypes.byref(n)))
    out = torch.empty((int(vocab), cols), dtype=d.dtype, device=d.device)
    ws = _workspace(n.value)
    _check(lib, lib.jorge_embedding_backward(d.data_ptr(), _ld(d), tok.data_ptr(), count, DTYPES[d.dtype], int(vocab),
                                             cols, float(scale), -1 if padding is None else int(padding),
                                             out.data_ptr(), cols, _ptr(ws), n.value, _stream(d)))
    return out


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, table, scale, padding):
        ctx.save_for_backward(tokens)
        ctx.more = (table.shape[0], scale, padding)
        return embedding_forward(tokens, table, scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        (tokens,), (vocab, scale, padding) = ctx.saved_tensors, ctx.more
        return None, embedding_backward(dout, tokens, vocab, scale, padding), None, None


def embedding(tokens, table, scale=1.0, padding=None):
    """Differentiable scale * table[tokens]; the gradient of table is dense (see embedding_backward)."""
    return _Embedding.apply(tokens, table, scale, padding)


# ---------------------------------------------------------------- cross entropy
LOSS_MAX_STRIDE = 1 << 22                     # JORGE_LOSS_MAX_STRIDE


def _loss_matrix(t, what, gradients):
    """_matrix, copied to dense rows where the row stride is more than the call takes, or, as its gradient will be
    written in that stride, than twice the width."""
    m = _matrix(t, what)
    most = 2 * m.shape[1] if gradients else LOSS_MAX_STRIDE
    return m.contiguous() if m.shape[0] > 1 and m.stride(0) > most else m


def _loss_args(hidden, weight, targets, ignore_index, label_smoothing, gradients=False):
    h, w = _loss_matrix(hidden, "hidden", gradients), _loss_matrix(weight, "weight", gradients)
    t = _int64s(targets, "targets")
    if weight.dim() != 2 or h.shape[1] != w.shape[1]:
        raise ValueError("weight: a matrix with a row of hidden's width per word is needed")
    if h.dtype != w.dtype:
        raise ValueError("hidden and weight must have one type")
    if tuple(targets.shape) != tuple(hidden.shape[:-1]):
        raise ValueError(f"targets: shape {tuple(targets.shape)} for hidden of shape {tuple(hidden.shape)}")
    shape = LossShape(h.shape[0], h.shape[1], w.shape[0], _ld(h), _ld(w), DTYPES[h.dtype], 0, int(ignore_index),
                      float(label_smoothing))
    return h, w, t, shape


def cross_entropy_forward(hidden, weight, targets, ignore_index=-100, label_smoothing=0.0):
    """(loss, lse, total) of the cross entropy of the logits hidden @ weight.T, which are not kept:
    loss and lse (log sum exp) one per row in fp32, total = [sum of the losses, rows with a target,
    mean over those (0 without any)]. Targets outside [0, vocab), or equal to ignore_index, are none."""
    lib = load_operators()
    h, w, t, shape = _loss_args(hidden, weight, targets, ignore_index, label_smoothing)
    n = _I64(0)
    _check(lib, lib.jorge_cross_entropy_workspace(ctypes.byref(shape), 0, ctypes.byref(n)))
    ws = _workspace(n.value)
    loss = torch.empty(targets.shape, dtype=torch.float32, device=h.device)
    lse = torch.empty(targets.shape, dtype=torch.float32, device=h.device)
    total = torch.empty(3, dtype=torch.float32, device=h.device)
    _check(lib, lib.jorge_cross_entropy_forward(ctypes.byref(shape), h.data_ptr(), w.data_ptr(), t.data_ptr(),
                                                loss.data_ptr(), lse.data_ptr(), total.data_ptr(), _ptr(ws), n.value,
                                                _stream(h)))
    return loss, lse, total


def cross_entropy_backward(grad, hidden, weight, targets, lse, total, reduction="mean", ignore_index=-100,
                           label_smoothing=0.0, need_hidden=True, need_weight=True):
    """(dhidden, dweight) from lse and total of cross_entropy_forward. grad: the gradient of every row's
    loss (reduction "none"), or of their sum or mean (one number, on the device)."""
    lib = load_operators()
    h, w, t, shape = _loss_args(hidden, weight, targets, ignore_index, label_smoothing, gradients=True)
    kind = REDUCTIONS[reduction]
    g = _cuda(grad, "grad").float().contiguous()
    if g.numel() != (h.shape[0] if kind == 0 else 1):
        raise ValueError("grad: one number per row for reduction 'none', one in all otherwise")
    for s, k, what in ((lse, h.shape[0], "lse"), (total, 3, "total")):
        if _cuda(s, what, (torch.float32,)).numel() != k or not s.is_contiguous():
            raise ValueError(f"{what}: as cross_entropy_forward returned it")
    n = _I64(0)
    _check(lib, lib.jorge_cross_entropy_workspace(ctypes.byref(shape), 1, ctypes.byref(n)))
    ws = _workspace(n.value)
    # In the matrices' own row strides, as the call writes them.
    dh = torch.empty((h.shape[0], shape.ldh), dtype=h.dtype, device=h.device) if need_hidden else None
    dw = torch.empty((w.shape[0], shape.ldw), dtype=w.dtype, device=w.device) if need_weight else None
    _check(lib, lib.jorge_cross_entropy_backward(ctypes.byref(shape), g.data_ptr(), kind, h.data_ptr(), w.data_ptr(),
                                                 t.data_ptr(), lse.data_ptr(), total.data_ptr(), _ptr(dh), _ptr(dw),
                                                 _ptr(ws), n.value, _stream(h)))
    if need_hidden:
        dh = dh[:, :h.shape[1]].reshape(hidden.shape)
    return dh, dw[:, :w.shape[1]] if need_weight else None


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, ignore_index, label_smoothing, reduction):
        loss, lse, total = cross_entropy_forward(hidden, weight, targets, ignore_index, label_smoothing)
        ctx.save_for_backward(hidden, weight, targets, lse, total)
        ctx.more = (reduction, ignore_index, label_smoothing)
        return loss if reduction == "none" else total[0 if reduction == "sum" else 2].clone()

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        dh, dw = cross_entropy_backward(grad, *ctx.saved_tensors, *ctx.more, need_hidden=ctx.needs_input_grad[0],
                                        need_weight=ctx.needs_input_grad[1])
        return dh, dw, None, None, None, None


def linear_cross_entropy(hidden, weight, targets, ignore_index=-100, label_smoothing=0.0, reduction="mean"):
    """Differentiable cross entropy of hidden @ weight.T without the logits (see cross_entropy_forward).
    reduction: "mean" over the rows with a target, "sum" or "none"."""
    if reduction not in REDUCTIONS:
        raise ValueError(f"reduction: {reduction!r} is none of {sorted(REDUCTIONS)}")
    return _CrossEntropy.apply(hidden, weight, targets, ignore_index, label_smoothing, reduction)


# ---------------------------------------------------------------- AdamW
def _gradient_norm(lib, tensors, count, max_norm):
    n = _I64(0)
    _check(lib, lib.jorge_gradient_norm_workspace(tensors, count, ctypes.byref(n)))
    ws, out = _workspace(n.value), torch.empty(2, dtype=torch.float32, device="cuda")
    _check(lib, lib.jorge_gradient_norm(tensors, count, float(max_norm), out.data_ptr(), _ptr(ws), n.value,
                                        _stream()))
    return out


def gradient_norm(grads, max_norm=0.0):
    """[norm, factor] on the device: the root of the sum of all gradients' squares, and what scales them
    to max_norm where that is positive and below it (else 1). grads: fp32 or bfloat16, None entries are left out."""
    grads = [_cuda(g, "gradient") for g in grads if g is not None]
    grads = [g if _dense(g) else g.contiguous() for g in grads]
    tensors = (AdamWTensor * max(1, len(grads)))(*[AdamWTensor(0, g.data_ptr(), g.numel(), 0, DTYPES[g.dtype], 0)
                                                   for g in grads])
    return _gradient_norm(load_operators(), tensors, len(grads), max_norm)


class AdamW:
    """AdamW steps of a list of dense fp32 or bfloat16 CUDA tensors, all in one launch (per 112 of them).

    bits: 32, or 8 for moments of a byte per element with a scale per block of 256, rounded by random
    bits made from seed, the step and the element's place (include/jorge_lm.h has the format). moments:
    existing flat buffers to take over instead of zeros, as `moments` of another AdamW over tensors of
    the same sizes. steps: of each tensor, the steps it has taken; a tensor without a gradient takes none, and
    its bias corrections (and random bits) go by its own count. t: the most of them; setting it sets them all.
    norm: after a step with max_norm, the gradients' global norm before clipping (a device tensor).

    A step captured into a graph is one step for good: replays repeat its count, rates and random bits, and
    advance nothing here. Capture the passes of a training step, and take the step itself outside; a warning
    says so at a capture.
    """

    def __init__(self, params, bits=32, seed=0, moments=None):
        self.lib = load_operators()
        self.params = list(params)
        self.bits, self.seed, self.t, self.norm = int(bits), int(seed), 0, None
        if self.bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        if not 0 <= self.seed < 1 << 32:
            raise ValueError("seed must be in [0, 2^32)")
        for i, p in enumerate(self.params):
            if not _dense(_cuda(p, f"parameter {i}")):
                raise ValueError(f"parameter {i}: a dense tensor is needed")
        spans = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()) for p in self.params if p.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("parameters: no two may share memory (both would be stepped at once)")
        self._numel = [p.numel() for p in self.params]
        self._layout = [(p.dtype, p.shape, p.stride(), p.get_device()) for p in self.params]
        self.blocks = np.cumsum([0] + [-(-n // BLOCK) for n in self._numel])
        self._tensors = (AdamWTensor * max(1, len(self.params)))()
        self._table = np.frombuffer(self._tensors, dtype=np.dtype(AdamWTensor))[:len(self.params)]
        self._table["numel"] = self._numel
        self._table["block"] = self.blocks[:-1]
        self._table["dtype"] = [DTYPES[p.dtype] for p in self.params]
        total = int(self.blocks[-1])
        kind = torch.float32 if self.bits == 32 else torch.uint8
        want = {"exp_avg": (kind, total * BLOCK), "exp_avg_sq": (kind, total * BLOCK)}
        if self.bits == 8:
            want.update(exp_avg_scale=(torch.uint8, total), exp_avg_sq_scale=(torch.uint8, total))
        if moments is None:
            moments = {k: torch.zeros(n, dtype=d, device="cuda") for k, (d, n) in want.items()}
        for k, (d, n) in want.items():
            m = moments.get(k)
            if m is None or _cuda(m, k, (d,)).shape != (n,) or not m.is_contiguous():
                raise ValueError(f"{k}: a dense tensor of {n} elements of {d} is needed")
        self.moments = {k: moments[k] for k in want}
        self._moments = AdamWMoments(*(_ptr(self.moments.get(k)) for k in (
            "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")), total, self.bits, self.seed)

    @property
    def t(self):
        return self._t if self._steps is None else max(self._steps)

    @t.setter
    def t(self, value):
        self._t, self._steps = int(value), None               # _steps: one count each, where they differ

    @property
    def steps(self):
        return [self._t] * len(self.params) if self._steps is None else list(self._steps)

    def _gradients(self, grads):
        """Puts the gradients' pointers into the table; a parameter without one (None) takes no part. Returns
        temporaries to keep until the launch, and whether every parameter takes part."""
        if len(grads) != len(self.params):
            raise ValueError(f"grads: expected {len(self.params)} tensors, got {len(grads)}")
        keep, ptrs, numel = [], [], self._numel
        for i, (g, (dtype, shape, stride, device)) in enumerate(zip(grads, self._layout)):
            if g is None:
                if numel is self._numel:
                    numel = list(numel)
                numel[i] = 0
                ptrs.append(0)
                continue
            if g.dtype is not dtype or g.shape != shape or g.get_device() != device:
                raise ValueError("grads: each must have its parameter's shape, type and device")
            if g.stride() != stride:
                g = torch.empty_strided(shape, stride, dtype=dtype, device=g.device).copy_(g)
                keep.append(g)
            ptrs.append(g.data_ptr())
        self._table["grad"] = ptrs
        self._table["numel"] = numel
        return keep, numel is self._numel

    def step(self, grads=None, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, max_norm=0.0, clip=None):
        """One step from the gradients (default: each parameter's .grad; None entries are left as they
        are). max_norm > 0 scales all gradients to that global norm if theirs is larger; clip: the factor
        itself, one fp32 number on the device (of another gradient_norm call)."""
        grads = [p.grad for p in self.params] if grads is None else grads
        keep, whole = self._gradients(grads)
        for p, (dtype, shape, stride, device) in zip(self.params, self._layout):
            if p.dtype is not dtype or p.get_device() != device or p.shape != shape or p.stride() != stride:
                raise ValueError("a parameter's type, device, shape or layout has changed since it was handed over")
        self._table["param"] = [p.data_ptr() for p in self.params]
        if max_norm and clip is not None:
            raise ValueError("max_norm or clip, not both")
        if max_norm:
            out = _gradient_norm(self.lib, self._tensors, len(self.params), max_norm)
            self.norm, clip = out[0], out[1:]
        elif clip is not None and (_cuda(clip, "clip", (torch.float32,)).numel() != 1):
            raise ValueError("clip: one number is needed")
        if torch.cuda.is_current_stream_capturing():
            warnings.warn("a captured AdamW step repeats its own step count, rates and random bits at every replay")
        hyper = (float(lr), float(beta1), float(beta2), float(eps), float(weight_decay), _ptr(clip), _stream())
        if whole and self._steps is None:
            self._launch(self._t + 1, hyper)
            self._t += 1
        else:
            steps = self.steps
            given = [i for i, g in enumerate(grads) if g is not None]
            counts = sorted({steps[i] for i in given}) or [self.t]
            if len(counts) > 1:
                numel = self._table["numel"].copy()
            for t in counts:                                  # a call for each count of steps among the tensors
                if len(counts) > 1:
                    part = [i for i in given if steps[i] == t]
                    self._table["numel"] = 0
                    self._table["numel"][part] = numel[part]
                self._launch(t + 1, hyper)
            for i in given:
                steps[i] += 1
            self._t, self._steps = (steps[0], None) if len(set(steps)) == 1 else (None, steps)
        # What autograd saved of a parameter no longer holds: a backward pass that needs it has to say so.
        torch.autograd.graph.increment_version(
            self.params if whole else [p for p, g in zip(self.params, grads) if g is not None])
        del keep

    def _launch(self, t, hyper):
        """Step t of the table's tensors."""
        _check(self.lib, self.lib.jorge_adamw_step(self._tensors, len(self.params), ctypes.byref(self._moments), t,
                                                   *hyper))

    def gradient_norm(self, grads=None, max_norm=0.0):
        """[norm, clip factor] of the gradients on the device, without a step (see gradient_norm)."""
        keep, _ = self._gradients([p.grad for p in self.params] if grads is None else grads)
        out = _gradient_norm(self.lib, self._tensors, len(self.params), max_norm)
        del keep
        return out

    def moment_values(self, dtype=torch.float32):
        """The two moments' values as new flat tensors of dtype, in the layout of `moments` (parameter i starts
        at blocks[i] * 256)."""
        if self.bits == 32:
            return tuple(self.moments[k].to(dtype, copy=True) for k in ("exp_avg", "exp_avg_sq"))
        total, out = int(self.blocks[-1]), []
        for second in (0, 1):
            v = torch.empty(total * BLOCK, dtype=dtype, device="cuda")
            _check(self.lib, self.lib.jorge_adamw_read(ctypes.byref(self._moments), second, 0, total, v.data_ptr(),
                                                       DTYPES[dtype], _stream()))
            out.append(v)
        return out[0], out[1]

    def set_moment_values(self, exp_avg, exp_avg_sq):
        """Takes the moments' values from flat fp32 tensors in the layout of moment_values (8 bits: rounded to
        nearest)."""
        values = {"exp_avg": exp_avg, "exp_avg_sq": exp_avg_sq}
        for k, v in values.items():
            values[k] = _cuda(v, k, (torch.float32,)).contiguous()
            if v.shape != self.moments[k].shape:
                raise ValueError(f"{k}: {self.moments[k].numel()} values are needed")
        for second, (k, v) in enumerate(values.items()):
            if self.bits == 32:
                self.moments[k].copy_(v)
            else:
                _check(self.lib, self.lib.jorge_adamw_write(ctypes.byref(self._moments), second, 0,
                                                            int(self.blocks[-1]), v.data_ptr(), _stream()))

    def state_dict(self):
        return {"t": self.t, "steps": self.steps, "bits": self.bits, "seed": self.seed,
                **{k: v.cpu() for k, v in self.moments.items()}}

    def check_state_dict(self, sd):
        """Raises ValueError unless load_state_dict would take sd whole."""
        held = all(isinstance(sd.get(k), torch.Tensor) and sd[k].shape == v.shape for k, v in self.moments.items())
        if not held or sd.get("bits") != self.bits or len(sd.get("steps", self.params)) != len(self.params):
            raise ValueError("the state is of another set of tensors or of other bits")
        if not all(int(t) >= 0 for t in [sd.get("t", -1), *sd.get("steps", [])]):
            raise ValueError("the state holds no count of steps")
        if not 0 <= int(sd.get("seed", -1)) < 1 << 32:
            raise ValueError("the state's seed must be in [0, 2^32)")

    def load_state_dict(self, sd):
        """Takes over what state_dict returned (its moments are copied); changes nothing if it is refused."""
        self.check_state_dict(sd)
        for k, v in self.moments.items():
            v.copy_(sd[k])
        self.t, self.seed = int(sd["t"]), int(sd["seed"])
        self._moments.seed = self.seed
        steps = [int(t) for t in sd.get("steps", [])]         # absent: all tensors took t steps
        if len(set(steps)) > 1:
            self._t, self._steps = None, steps


def _dense(t):
    """Whether t's elements fill one span of memory without overlap, in whatever order of dimensions."""
    expect = 1
    for n, s in sorted(((n, s) for n, s in zip(t.shape, t.stride()) if n > 1), key=lambda x: x[1]):
        if s != expect:
            return False
        expect *= n
    return True
