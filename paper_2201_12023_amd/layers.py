"""Thin ctypes binding over the C ABI in ``include/alpa_layers.h`` (argument marshalling, and nodes of torch's graph): the
products of dense and expert layers and the loss over a vocabulary, forward and backward.

Same names as the C entry points.  Arguments and results are torch tensors on one GPU; results and work memory come from
torch's allocator, every step runs in the HIP kernels of ``libalpa_dp.so``.  Work is queued on ``stream`` (a
torch.cuda.Stream; the current one if None) and not waited for; tensors that belong to another stream are the caller's to
order and to keep.  The last dimension of a tensor must be contiguous, rows may be
any distance apart.

The forward calls can be differentiated: where an argument requires a gradient their results are part of torch's graph, and its backward
pass makes the calls of this module.  What is kept for those, z and lse, can not be: a loss that depends on them raises an error in the
backward pass.  The backward calls themselves record nothing.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.function import once_differentiable

from . import binding

ALPA_F32, ALPA_F16, ALPA_BF16 = 0, 1, 2
ALPA_ACT_NONE, ALPA_ACT_RELU, ALPA_ACT_GELU, ALPA_ACT_GELU_TANH, ALPA_ACT_SILU = range(5)
MAX_WIDTH = 1 << 20
MAX_ROWS = 1 << 28
MAX_EXPERTS = 4096
MAX_WORDS = 1 << 24
_TYPES = {torch.float32: ALPA_F32, torch.float16: ALPA_F16, torch.bfloat16: ALPA_BF16}

SYMBOLS = ["alpa_linear_forward", "alpa_linear_forward_work", "alpa_linear_backward", "alpa_linear_backward_work",
           "alpa_experts_forward", "alpa_experts_forward_work", "alpa_experts_backward", "alpa_experts_backward_work",
           "alpa_vocab_loss_forward", "alpa_vocab_loss_forward_work", "alpa_vocab_loss_backward",
           "alpa_vocab_loss_backward_work"]


class alpa_mat_t(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("ld", ctypes.c_int64)]


_ready = None


def load():
    """The library with the argument types of the layer operators set (raises if it is not built)."""
    global _ready
    if _ready is not None:
        return _ready
    L = binding.load()
    i, n, vp, mat = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, alpa_mat_t
    L.alpa_linear_forward.argtypes = [i, i, n, n, n, mat, mat, vp, mat, mat, mat, vp, n, vp]
    L.alpa_linear_backward.argtypes = [i, i, n, n, n, mat, mat, mat, mat, mat, mat, vp, vp, n, vp]
    L.alpa_experts_forward.argtypes = [i, i, n, i, n, n, vp, mat, mat, vp, mat, mat, mat, vp, n, vp]
    L.alpa_experts_backward.argtypes = [i, i, n, i, n, n, vp, mat, mat, mat, mat, mat, mat, vp, vp, n, vp]
    L.alpa_vocab_loss_forward.argtypes = [i, n, n, n, mat, mat, vp, vp, vp, vp, n, vp]
    L.alpa_vocab_loss_backward.argtypes = [i, n, n, n, vp, mat, mat, vp, vp, mat, mat, vp, n, vp]
    L.alpa_linear_forward_work.argtypes = [i, n, n, n, mat, mat]
    L.alpa_linear_backward_work.argtypes = [i, i, n, n, n, mat, mat, mat]
    L.alpa_experts_forward_work.argtypes = [i, n, i, n, n, mat, mat]
    L.alpa_experts_backward_work.argtypes = [i, i, n, i, n, n, mat, mat, mat]
    L.alpa_vocab_loss_forward_work.argtypes = [i, n, n, n, mat, mat]
    L.alpa_vocab_loss_backward_work.argtypes = [i, n, n, n, mat, mat]
    for s in SYMBOLS:
        getattr(L, s).restype = ctypes.c_int64 if s.endswith("_work") else ctypes.c_int
    _ready = L
    return L


def _type(x):
    if x.dtype not in _TYPES:
        raise ValueError(f"type {x.dtype} is not one of float32, float16, bfloat16")
    return _TYPES[x.dtype]


def _check(name, t, shape, dtype, device):
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} is {t.dtype} on {t.device}; {dtype} on {device} expected")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, {tuple(shape)} expected")


_NONE = alpa_mat_t(None, 0)


def _mat(name, t, shape, dtype, device):
    """A matrix, or matrices one behind the other, as the library takes it: its rows `ld` apart."""
    if t is None:
        return _NONE
    _check(name, t, shape, dtype, device)
    rows, n = shape[-2], shape[-1]
    if t.is_contiguous():
        return alpa_mat_t(t.data_ptr(), n)
    ld = t.stride(-2) if rows > 1 else n
    if len(shape) == 3 and rows == 1 and shape[0] > 1:
        ld = t.stride(0)
    if (n > 1 and t.stride(-1) != 1) or ld < n or (len(shape) == 3 and shape[0] > 1 and t.stride(0) != rows * ld):
        raise ValueError(f"{name} must have contiguous rows that do not overlap, experts one behind the other; "
                         f"strides are {tuple(t.stride())}")
    return alpa_mat_t(t.data_ptr(), ld)


def _new(t):
    """A result, contiguous as it was allocated."""
    return _NONE if t is None else alpa_mat_t(t.data_ptr(), t.shape[-1])


def _vec(name, t, shape, dtype, device):
    if t is None:
        return None
    _check(name, t, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


class _On:
    """The tensors' device and the stream of the call, as torch's current ones, so that results and work memory
    belong to that stream.  (Entering a context costs 6 us of the host's time: not done where nothing would change.)"""

    def __init__(self, x, stream):
        device = x.device
        if device.type != "cuda":
            raise ValueError("tensors must be on a GPU")
        self.context = None
        if stream is None:
            stream = torch.cuda.current_stream(device)
            if device.index != torch.cuda.current_device():
                self.context = torch.cuda.device(device)
        else:
            if stream.device != device:
                raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
            self.context = torch.cuda.stream(stream)
        self.raw = stream.cuda_stream

    def __enter__(self):
        if self.context is not None:
            self.context.__enter__()
        return self.raw

    def __exit__(self, *a):
        if self.context is not None:
            self.context.__exit__(*a)


def _work(need, device):
    """(tensor that keeps the memory, pointer, bytes)"""
    if need == 0:
        return None, None, 0
    t = torch.empty(need, dtype=torch.uint8, device=device)
    return t, t.data_ptr(), need


def _two(name, x):
    if x.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, not {x.dim()}")
    return x.shape


def _forward(x, w, offsets, bias, residual, act, keep_z, stream):
    L, d = load(), _type(x)
    rows, n_in = _two("x", x)
    n_out = w.shape[-2] if w.dim() >= 2 else 0
    dtype, device = x.dtype, x.device
    lead = () if offsets is None else (offsets.numel() - 1,)
    with _On(x, stream) as s:
        xm, wm = _mat("x", x, (rows, n_in), dtype, device), _mat("w", w, (*lead, n_out, n_in), dtype, device)
        b, r = _vec("bias", bias, (*lead, n_out), dtype, device), _mat("residual", residual, (rows, n_out), dtype, device)
        y = torch.empty((rows, n_out), dtype=dtype, device=device)
        z = torch.empty_like(y) if keep_z else None
        if offsets is None:
            keep, p, n = _work(L.alpa_linear_forward_work(d, rows, n_in, n_out, xm, wm), device)
            rc = L.alpa_linear_forward(d, act, rows, n_in, n_out, xm, wm, b, r, _new(y), _new(z), p, n, s)
        else:
            off = _vec("offsets", offsets, (lead[0] + 1,), torch.int32, device)
            keep, p, n = _work(L.alpa_experts_forward_work(d, rows, lead[0], n_in, n_out, xm, wm), device)
            rc = L.alpa_experts_forward(d, act, rows, lead[0], n_in, n_out, off, xm, wm, b, r, _new(y), _new(z), p, n, s)
        binding._check(rc)
    return (y, z) if keep_z else y


def _backward(dy, x, w, offsets, z, act, need, stream):
    L, d = load(), _type(dy)
    if not set(need) <= {"x", "w", "bias"}:
        raise ValueError(f"need is {need!r}: names out of 'x', 'w', 'bias' expected")
    rows, n_out = _two("dy", dy)
    if x is None and w is None:
        raise ValueError("one of x and w has to be given")
    n_in = (w if x is None else x).shape[-1]
    dtype, device = dy.dtype, dy.device
    lead = () if offsets is None else (offsets.numel() - 1,)
    with _On(dy, stream) as s:
        dym, zm = _mat("dy", dy, (rows, n_out), dtype, device), _mat("z", z, (rows, n_out), dtype, device)
        xm, wm = _mat("x", x, (rows, n_in), dtype, device), _mat("w", w, (*lead, n_out, n_in), dtype, device)
        new = lambda *size: torch.empty(size, dtype=dtype, device=device)
        dx = new(rows, n_in) if "x" in need else None
        dw = new(*lead, n_out, n_in) if "w" in need else None
        db = new(*lead, n_out) if "bias" in need else None
        bias = None if db is None else db.data_ptr()
        if offsets is None:
            keep, p, n = _work(L.alpa_linear_backward_work(d, act, rows, n_in, n_out, dym, xm, wm), device)
            rc = L.alpa_linear_backward(d, act, rows, n_in, n_out, dym, zm, xm, wm, _new(dx), _new(dw), bias, p, n, s)
        else:
            off = _vec("offsets", offsets, (lead[0] + 1,), torch.int32, device)
            keep, p, n = _work(L.alpa_experts_backward_work(d, act, rows, lead[0], n_in, n_out, dym, xm, wm), device)
            rc = L.alpa_experts_backward(d, act, rows, lead[0], n_in, n_out, off, dym, zm, xm, wm, _new(dx), _new(dw),
                                         bias, p, n, s)
        binding._check(rc)
    return dx, dw, db


def _recorded(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _apply(function, stream, *args):
    """The call as a node of torch's graph, whose backward pass runs on the stream that is current here."""
    if stream is None:
        return function.apply(*args, None)
    with torch.cuda.stream(stream):
        return function.apply(*args, stream)


class _Product(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, offsets, bias, residual, act, keep_z, stream):
        needs = ctx.needs_input_grad
        ctx.need = tuple(name for name, wanted in (("x", needs[0]), ("w", needs[1]), ("bias", needs[3])) if wanted)
        ctx.act = act
        has_z = keep_z or (act != ALPA_ACT_NONE and bool(ctx.need))
        result = _forward(x, w, offsets, bias, residual, act, has_z, stream)
        y, z = result if has_z else (result, None)
        # (of x and w one at least, for the sizes)
        ctx.save_for_backward(x if needs[1] or (ctx.need and not needs[0]) else None, w if needs[0] else None, offsets,
                              z if act != ALPA_ACT_NONE else None)
        ctx.set_materialize_grads(False)
        return (y, z) if keep_z else y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dz=None):
        if dz is not None:
            raise RuntimeError("z has no gradient: a loss may depend on y alone")
        if dy is None:
            return (None,) * 8
        x, w, offsets, z = ctx.saved_tensors
        dy = dy.contiguous()
        dx, dw, db = _backward(dy, x, w, offsets, z, ctx.act, ctx.need, None) if ctx.need else (None, None, None)
        dr = dy if ctx.needs_input_grad[4] else None
        if dr is not None and offsets is not None:
            row = torch.arange(dy.shape[0], device=dy.device)         # (rows of no expert do not have the residual)
            dr = torch.where(((row >= offsets[0]) & (row < offsets[-1]))[:, None], dy, torch.zeros_like(dy))
        return dx, dw, None, db, dr, None, None, None


class _VocabLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, target, stream):
        loss, lse = _vocab_loss(x, w, target, stream)
        ctx.save_for_backward(x, w, target, lse)
        ctx.set_materialize_grads(False)
        return loss, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss, dlse):
        if dlse is not None:
            raise RuntimeError("lse has no gradient: a loss may depend on the rows' losses alone")
        if dloss is None:
            return (None,) * 4
        x, w, target, lse = ctx.saved_tensors
        need = tuple(name for name, wanted in zip(("x", "w"), ctx.needs_input_grad) if wanted)
        return *alpa_vocab_loss_backward(dloss.contiguous(), x, w, target, lse, need), None, None


def alpa_linear_forward(x, w, bias=None, residual=None, act=ALPA_ACT_NONE, keep_z=False, stream=None):
    """act(x w^T + bias) + residual for x [rows, in], w [out, in]; with ``keep_z`` also what stands in front of the
    activation, which the backward pass takes: (y, z)."""
    if _recorded(x, w, bias, residual):
        return _apply(_Product, stream, x, w, None, bias, residual, act, keep_z)
    return _forward(x, w, None, bias, residual, act, keep_z, stream)


def alpa_linear_backward(dy, x, w, z=None, act=ALPA_ACT_NONE, need=("x", "w", "bias"), stream=None):
    """(dx, dw, dbias), None for those not in ``need``; x is only read for dw, w for dx, z for an activation."""
    return _backward(dy, x, w, None, z, act, need, stream)


def alpa_experts_forward(x, w, offsets, bias=None, residual=None, act=ALPA_ACT_NONE, keep_z=False, stream=None):
    """The same for rows sorted by expert: rows offsets[e] .. offsets[e + 1] - 1 (int32 tensor [experts + 1] on the GPU)
    through w[e] of [experts, out, in] and bias[e]; rows of no expert give zeros."""
    if _recorded(x, w, bias, residual):
        return _apply(_Product, stream, x, w, offsets, bias, residual, act, keep_z)
    return _forward(x, w, offsets, bias, residual, act, keep_z, stream)


def alpa_experts_backward(dy, x, w, offsets, z=None, act=ALPA_ACT_NONE, need=("x", "w", "bias"), stream=None):
    """(dx, dw, dbias) of alpa_experts_forward; an expert without rows gets zeros."""
    return _backward(dy, x, w, offsets, z, act, need, stream)


def _vocab_loss(x, w, target, stream):
    L, d = load(), _type(x)
    rows, n_in = _two("x", x)
    words = _two("w", w)[0]
    dtype, device = x.dtype, x.device
    with _On(x, stream) as s:
        xm, wm = _mat("x", x, (rows, n_in), dtype, device), _mat("w", w, (words, n_in), dtype, device)
        t = _vec("target", target, (rows,), torch.int64, device)
        loss = torch.empty((rows,), dtype=torch.float32, device=device)
        lse = torch.empty_like(loss)
        keep, p, n = _work(L.alpa_vocab_loss_forward_work(d, rows, n_in, words, xm, wm), device)
        binding._check(L.alpa_vocab_loss_forward(d, rows, n_in, words, xm, wm, t, loss.data_ptr(), lse.data_ptr(), p, n, s))
    return loss, lse


def alpa_vocab_loss_forward(x, w, target, stream=None):
    """(loss, lse), float32 [rows]: cross entropy of softmax(x w^T) for x [rows, in], w [words, in], target int64 [rows];
    a negative target leaves the row out (loss 0).  ``lse`` is what the backward pass takes."""
    if _recorded(x, w):
        return _apply(_VocabLoss, stream, x, w, target)
    return _vocab_loss(x, w, target, stream)


def alpa_vocab_loss_backward(dloss, x, w, target, lse, need=("x", "w"), stream=None):
    """(dx, dw) for the rows' loss gradients (float32 [rows]), None for those not in ``need``."""
    L, d = load(), _type(x)
    if not set(need) <= {"x", "w"}:
        raise ValueError(f"need is {need!r}: names out of 'x', 'w' expected")
    rows, n_in = _two("x", x)
    words = _two("w", w)[0]
    dtype, device = x.dtype, x.device
    with _On(x, stream) as s:
        xm, wm = _mat("x", x, (rows, n_in), dtype, device), _mat("w", w, (words, n_in), dtype, device)
        t = _vec("target", target, (rows,), torch.int64, device)
        g, l = (_vec(k, v, (rows,), torch.float32, device) for k, v in (("dloss", dloss), ("lse", lse)))
        dx = torch.empty((rows, n_in), dtype=dtype, device=device) if "x" in need else None
        dw = torch.empty((words, n_in), dtype=dtype, device=device) if "w" in need else None
        keep, p, n = _work(L.alpa_vocab_loss_backward_work(d, rows, n_in, words, xm, wm), device)
        binding._check(L.alpa_vocab_loss_backward(d, rows, n_in, words, g, xm, wm, t, l, _new(dx), _new(dw), p, n, s))
    return dx, dw
