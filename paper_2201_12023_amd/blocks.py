"""Thin ctypes binding over the C ABI in ``include/alpa_blocks.h`` (argument marshalling, and nodes of torch's graph): what a block has
between its products, which are in ``layers``: attention, rotary positions and layer norm, forward and backward.

Same names as the C entry points, same manner as ``layers``: torch tensors on one GPU, results and work memory from torch's allocator, work queued on
``stream`` (a torch.cuda.Stream; the current one if None) and not waited for.  The last dimension of a tensor must be contiguous, rows and heads may
be any distance apart, so that queries, keys and values may be slices of one product's result.  A result that is given must not overlap another tensor of
the call, but for x where rotary positions turn it in place.

The forward calls can be differentiated: where an argument requires a gradient their results are part of torch's graph, and its backward pass makes
the calls of this module.  What is kept for those (lse; mean and rstd) has no gradient: a loss that depends on it raises an error in the backward pass.
The backward calls themselves record nothing.  There are no forward-mode derivatives: tensors that have one are refused.  All calls may be recorded into a
HIP graph; a backward pass of torch's graph only if that graph was built in the same recording.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd.function import once_differentiable

from . import binding
from . import layers as _l

MAX_HEADS = 4096
MAX_DIM = 4096
ATTENTION_MAX_DIM = 256
ATTENTION_MAX_SEQS = 65536
ATTENTION_MAX_ITEMS = 1 << 30

SYMBOLS = ["alpa_attention_forward", "alpa_attention_forward_work", "alpa_attention_backward", "alpa_attention_backward_work",
           "alpa_rotary_forward", "alpa_rotary_backward", "alpa_rotary_frequencies",
           "alpa_norm_forward", "alpa_norm_backward", "alpa_norm_backward_work"]


class alpa_heads_t(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class alpa_attention_t(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("seqs", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("k_step", ctypes.c_int32), ("scale", ctypes.c_float), ("cap", ctypes.c_float),
                ("rows", ctypes.c_int64), ("k_rows", ctypes.c_int64), ("offsets", ctypes.c_void_p), ("k_offsets", ctypes.c_void_p),
                ("prefix", ctypes.c_void_p), ("slopes", ctypes.c_void_p)]


_ready = None


def load():
    """The library with the argument types of these calls set (raises if it is not built)."""
    global _ready
    if _ready is not None:
        return _ready
    L = binding.load()
    i, n, f, vp, mat, heads, how = (ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, _l.alpa_mat_t, alpa_heads_t,
                                    ctypes.POINTER(alpa_attention_t))
    L.alpa_attention_forward_work.argtypes = [how, heads, heads, heads]
    L.alpa_attention_forward.argtypes = [how, heads, heads, heads, heads, vp, vp, n, vp]
    L.alpa_attention_backward_work.argtypes = [how, heads, heads, heads, heads, heads]
    L.alpa_attention_backward.argtypes = [how, heads, heads, heads, heads, heads, vp, heads, heads, heads, vp, n, vp]
    L.alpa_rotary_forward.argtypes = L.alpa_rotary_backward.argtypes = [i, n, i, i, i, i, f, vp, vp, heads, heads, vp]
    L.alpa_rotary_frequencies.argtypes = [i] + [ctypes.c_double] * 5 + [vp]
    L.alpa_norm_forward.argtypes = [i, n, n, f, mat, vp, vp, mat, vp, vp, vp]
    L.alpa_norm_backward_work.argtypes = [i, n, n]
    L.alpa_norm_backward.argtypes = [i, n, n, mat, mat, vp, vp, vp, mat, vp, vp, vp, n, vp]
    for s in SYMBOLS:
        getattr(L, s).restype = ctypes.c_int64 if s.endswith("_work") else ctypes.c_int
    _ready = L
    return L


_NONE = alpa_heads_t(None, 0, 0)


def _on(call, x, stream, *args):
    """``call`` with the stream's handle and ``args``, the tensors' device and the stream being torch's current ones.  (Calls of a few microseconds of the GPU's
    time wait for the host: nothing is done here that would not change anything.)"""
    device = x.device
    _l._type(x)
    if stream is None and device.type == "cuda" and device.index == torch.cuda.current_device():
        return call(torch._C._cuda_getCurrentRawStream(device.index), *args)
    with _l._On(x, stream) as s:
        return call(s, *args)


def _vec(name, t, shape, dtype, device):
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device or t.shape != shape or not t.is_contiguous():
        return _l._vec(name, t, shape, dtype, device)              # (which says what is wrong)
    return t.data_ptr()


def _mat(name, t, shape, dtype, device):
    if t.dtype is not dtype or t.device != device or t.shape != shape or not t.is_contiguous():
        return _l._mat(name, t, shape, dtype, device)
    return _l.alpa_mat_t(t.data_ptr(), shape[1])


def _ptr(t):
    return None if t is None else t.data_ptr()


def _three(name, x):
    if x.dim() != 3:
        raise ValueError(f"{name} must have three dimensions, not {x.dim()}")
    return x.shape


def _heads(name, t, shape, dtype, device):
    """A tensor [rows, heads, dim] as the library takes it."""
    if t.dtype is not dtype or t.device != device or t.shape != shape:
        _l._check(name, t, shape, dtype, device)
    row, head, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError(f"{name} must have contiguous heads; strides are {(row, head, one)}")
    return alpa_heads_t(t.data_ptr(), row, head)


def _new(t):
    """A result, contiguous as it was allocated."""
    return _NONE if t is None else alpa_heads_t(t.data_ptr(), t.shape[1] * t.shape[2], t.shape[2])


def _written(*tensors):
    """Tells torch's graph that given tensors were written to, so that it refuses a backward pass that needs what they held (1 us of the host's time each)."""
    for t in tensors:
        if t is not None:
            torch.autograd.graph.increment_version(t)


# ------------------------------------------------------------------ attention

def _how(q, k, offsets, k_offsets, scale, cap, slopes, causal, prefix):
    """The alpa_attention_t of a call, which points into these tensors."""
    rows, heads, dim = _three("q", q)
    k_rows, kv_heads, _ = _three("k", k)
    device, ints = q.device, torch.int32
    if offsets is None and k_offsets is not None and k_offsets.numel() != 2:
        raise ValueError("k_offsets of several sequences are given without offsets")
    seqs = 1 if offsets is None else offsets.numel() - 1
    if k_offsets is None and offsets is not None:
        k_offsets = offsets
    pairs = k_offsets is not None and k_offsets.dim() == 2
    a = alpa_attention_t(_l._type(q), seqs, heads, kv_heads, dim, bool(causal), 2 if pairs else 1, dim ** -0.5 if scale is None else scale, cap,
                         rows, k_rows, _vec("offsets", offsets, (seqs + 1,), ints, device),
                         _vec("k_offsets", k_offsets, (seqs, 2) if pairs else (seqs + 1,), ints, device), _vec("prefix", prefix, (seqs,), ints, device),
                         _vec("slopes", slopes, (heads,), torch.float32, device))
    return a


def _attention(q, k, v, offsets, k_offsets, scale, cap, slopes, causal, prefix, keep_lse, stream):
    return _on(_attention_on, q, stream, q, k, v, offsets, k_offsets, scale, cap, slopes, causal, prefix, keep_lse)


def _attention_on(s, q, k, v, offsets, k_offsets, scale, cap, slopes, causal, prefix, keep_lse):
    L = _ready or load()
    a = _how(q, k, offsets, k_offsets, scale, cap, slopes, causal, prefix)
    shape, dtype, device = k.shape, q.dtype, q.device
    if shape[2] != a.dim:
        raise ValueError(f"k has heads of {shape[2]} elements, q of {a.dim}")
    qm, km, vm = _heads("q", q, q.shape, dtype, device), _heads("k", k, shape, dtype, device), _heads("v", v, shape, dtype, device)
    y = q.new_empty(q.shape)
    lse = q.new_empty(q.shape[:2], dtype=torch.float32) if keep_lse else None
    held, p, n = _l._work(L.alpa_attention_forward_work(a, qm, km, vm), device)
    binding._check(L.alpa_attention_forward(a, qm, km, vm, _new(y), _ptr(lse), p, n, s))
    return (y, lse) if keep_lse else y


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, offsets, k_offsets, slopes, prefix, how, keep_lse, stream):
        scale, cap, causal = how
        y, lse = _attention(q, k, v, offsets, k_offsets, scale, cap, slopes, causal, prefix, True, stream)
        ctx.save_for_backward(q, k, v, y, lse, offsets, k_offsets, slopes, prefix)
        ctx.how = how
        ctx.set_materialize_grads(False)
        return (y, lse) if keep_lse else y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dlse=None):
        if dlse is not None:
            raise RuntimeError("lse has no gradient: a loss may depend on y alone")
        if dy is None:
            return (None,) * 10
        q, k, v, y, lse, offsets, k_offsets, slopes, prefix = ctx.saved_tensors
        scale, cap, causal = ctx.how
        need = tuple(name for name, wanted in zip(("q", "k", "v"), ctx.needs_input_grad) if wanted)
        if dy.stride(2) != 1:
            dy = dy.contiguous()
        return *alpa_attention_backward(dy, q, k, v, y, lse, offsets, k_offsets, scale, cap, slopes, causal, prefix, need), *(None,) * 7


def alpa_attention_forward(q, k, v, offsets=None, k_offsets=None, scale=None, cap=0.0, slopes=None, causal=False, prefix=None, keep_lse=False,
                           stream=None):
    """Attention of packed sequences, for q [rows, heads, dim] and k, v [key rows, kv heads, dim]; with ``keep_lse`` also what the backward pass takes:
    (y, lse), float32 [rows, heads].

    offsets: int32 [seqs + 1] on the GPU, sequence s being rows offsets[s] .. offsets[s + 1] - 1 (None: one sequence of all rows).
    k_offsets: the same for keys (None: ``offsets``, with one sequence too, so that rows of none have keys of none; if that is None as well, all keys), or [seqs, 2],
    first key and end of each sequence in a cache with gaps.
    scale: of q k^T (None: dim ** -0.5).  cap: scores become cap * tanh(score / cap), 0 leaves them.  slopes: float32 [heads], the score's loss with each key of
    distance.  causal: a row sees keys up to its own place, the last row standing at the last key, and the first prefix[s] (int32 [seqs]) ones."""
    if _l._recorded(q, k, v, slopes):
        if slopes is not None and slopes.requires_grad:
            raise ValueError("slopes have no gradient")
        if k_offsets is not None and k_offsets.dim() == 2:
            raise ValueError("keys that are not packed have no gradient")
        return _l._apply(_Attention, stream, q, k, v, offsets, k_offsets, slopes, prefix, (scale, cap, causal), keep_lse)
    return _attention(q, k, v, offsets, k_offsets, scale, cap, slopes, causal, prefix, keep_lse, stream)


def alpa_attention_backward(dy, q, k, v, y, lse, offsets=None, k_offsets=None, scale=None, cap=0.0, slopes=None, causal=False, prefix=None,
                            need=("q", "k", "v"), out=None, stream=None):
    """(dq, dk, dv) of alpa_attention_forward, None for those not in ``need``; y and lse are its results.  ``out``: three tensors to put them in (None where
    one is not needed), such as the slices of one product's gradient."""
    _l._no_tangents(dy, q, k, v, y, lse)
    if not set(need) <= {"q", "k", "v"}:
        raise ValueError(f"need is {need!r}: names out of 'q', 'k', 'v' expected")
    if k_offsets is not None and k_offsets.dim() == 2:
        raise ValueError("keys that are not packed have no gradient")
    return _on(_attention_backward_on, q, stream, dy, q, k, v, y, lse, offsets, k_offsets, scale, cap, slopes, causal, prefix, need, out)


def _attention_backward_on(s, dy, q, k, v, y, lse, offsets, k_offsets, scale, cap, slopes, causal, prefix, need, out):
    L = _ready or load()
    a = _how(q, k, offsets, k_offsets, scale, cap, slopes, causal, prefix)
    shape, dtype, device = (a.k_rows, a.kv_heads, a.dim), q.dtype, q.device
    mats = [_heads(name, t, size, dtype, device) for name, t, size in (("dy", dy, q.shape), ("q", q, q.shape), ("k", k, shape), ("v", v, shape),
                                                                       ("y", y, q.shape))]
    l = _vec("lse", lse, q.shape[:2], torch.float32, device)
    sizes = (("q", q.shape), ("k", shape), ("v", shape))
    if out is None:
        grads = tuple(q.new_empty(size) if name in need else None for name, size in sizes)
        results = [_new(t) for t in grads]
    else:
        grads = tuple(t if name in need else None for t, (name, _) in zip(out, sizes))
        if any(t is None for t, (name, _) in zip(grads, sizes) if name in need):
            raise ValueError("out lacks a gradient that is needed")
        results = [_NONE if t is None else _heads("d" + name, t, size, dtype, device) for t, (name, size) in zip(grads, sizes)]
    held, p, n = _l._work(L.alpa_attention_backward_work(a, *mats), device)
    binding._check(L.alpa_attention_backward(a, *mats, l, *results, p, n, s))
    if out is not None:
        _written(*grads)
    return grads


# ------------------------------------------------------------------ rotary positions

def alpa_rotary_frequencies(rot, base=10000.0, factor=1.0, context=0.0, low=1.0, high=32.0, device="cuda"):
    """float64 [rot / 2]: base ** (-2 t / rot), for contexts ``factor`` times longer than those a model was trained on.  Pairs that turn ``high`` times and
    more over ``context`` positions stay, those that turn ``low`` times and less are divided by factor, those between linearly in between; context 0 divides
    all."""
    f = torch.empty(max(rot // 2, 1), dtype=torch.float64)
    binding._check(load().alpa_rotary_frequencies(rot, base, factor, context, low, high, f.data_ptr()))
    return f.to(device)


def _rotary(name, x, positions, frequencies, interleaved, scale, out, stream):
    return _on(_rotary_on, x, stream, name, x, positions, frequencies, interleaved, scale, out)


def _rotary_on(s, name, x, positions, frequencies, interleaved, scale, out):
    L = _ready or load()
    shape, dtype, device = _three("x", x), x.dtype, x.device
    xm, half = _heads("x", x, shape, dtype, device), frequencies.numel()
    p, f = _vec("positions", positions, shape[:1], torch.int64, device), _vec("frequencies", frequencies, (half,), torch.float64, device)
    y = x.new_empty(shape) if out is None else out
    ym = _new(y) if out is None else _heads("out", out, shape, dtype, device)
    binding._check(getattr(L, name)(_l._type(x), *shape, 2 * half, interleaved, scale, p, f, xm, ym, s))
    if out is not None:
        _written(out)
    return y


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, frequencies, interleaved, scale, stream):
        ctx.save_for_backward(positions, frequencies)
        ctx.how = interleaved, scale
        return _rotary("alpa_rotary_forward", x, positions, frequencies, interleaved, scale, None, stream)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        if dy.stride(2) != 1:
            dy = dy.contiguous()
        return alpa_rotary_backward(dy, *ctx.saved_tensors, *ctx.how), None, None, None, None, None


def alpa_rotary_forward(x, positions, frequencies, interleaved=False, scale=1.0, out=None, stream=None):
    """x [rows, heads, dim] with the first 2 * len(frequencies) elements of each head turned by positions (int64 [rows]) times frequencies (float64, radians) and
    scaled: pairs (t, t + half), or (2 t, 2 t + 1) if ``interleaved``.  ``out``: where to put it, x itself to turn it in place.  Frequencies are constants."""
    if _l._recorded(x, frequencies, out):
        if frequencies.requires_grad:
            raise ValueError("frequencies have no gradient")
        if out is not None:
            raise ValueError("a result that is given cannot be recorded")
        return _l._apply(_Rotary, stream, x, positions, frequencies, interleaved, scale)
    return _rotary("alpa_rotary_forward", x, positions, frequencies, interleaved, scale, out, stream)


def alpa_rotary_backward(dy, positions, frequencies, interleaved=False, scale=1.0, out=None, stream=None):
    """dx: the same turned the other way."""
    _l._no_tangents(dy, frequencies)
    return _rotary("alpa_rotary_backward", dy, positions, frequencies, interleaved, scale, out, stream)


# ------------------------------------------------------------------ layer norm

def _norm(x, weight, bias, eps, keep, stream):
    return _on(_norm_on, x, stream, x, weight, bias, eps, keep)


def _norm_on(s, x, weight, bias, eps, keep):
    L = _ready or load()
    shape, dtype, device = _l._two("x", x), x.dtype, x.device
    xm, w, b = _mat("x", x, shape, dtype, device), _vec("weight", weight, shape[1:], dtype, device), _vec("bias", bias, shape[1:], dtype, device)
    y = x.new_empty(shape)
    mean, rstd = (x.new_empty(shape[:1], dtype=torch.float32) for _ in range(2)) if keep else (None, None)
    binding._check(L.alpa_norm_forward(_l._type(x), *shape, eps, xm, w, b, _l._new(y), _ptr(mean), _ptr(rstd), s))
    return (y, mean, rstd) if keep else y


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, keep, stream):
        y, mean, rstd = _norm(x, weight, bias, eps, True, stream)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.set_materialize_grads(False)
        return (y, mean, rstd) if keep else y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dmean=None, drstd=None):
        if dmean is not None or drstd is not None:
            raise RuntimeError("mean and rstd have no gradient: a loss may depend on y alone")
        if dy is None:
            return (None,) * 6
        x, weight, mean, rstd = ctx.saved_tensors
        need = tuple(name for name, wanted in zip(("x", "weight", "bias"), ctx.needs_input_grad) if wanted)
        return *alpa_norm_backward(dy.contiguous(), x, mean, rstd, weight, need), None, None, None


def alpa_norm_forward(x, weight=None, bias=None, eps=1e-5, keep=False, stream=None):
    """(x - mean) * rstd * weight + bias for rows of x [rows, n], rstd = 1 / sqrt(variance + eps); with ``keep`` also what the backward pass takes:
    (y, mean, rstd), float32 [rows]."""
    if _l._recorded(x, weight, bias):
        return _l._apply(_Norm, stream, x, weight, bias, eps, keep)
    return _norm(x, weight, bias, eps, keep, stream)


def alpa_norm_backward(dy, x, mean, rstd, weight=None, need=("x", "weight", "bias"), stream=None):
    """(dx, dweight, dbias) of alpa_norm_forward, None for those not in ``need``."""
    _l._no_tangents(dy, x, mean, rstd, weight)
    if not set(need) <= {"x", "weight", "bias"}:
        raise ValueError(f"need is {need!r}: names out of 'x', 'weight', 'bias' expected")
    return _on(_norm_backward_on, x, stream, dy, x, mean, rstd, weight, need)


def _norm_backward_on(s, dy, x, mean, rstd, weight, need):
    L, d = _ready or load(), _l._type(x)
    shape, dtype, device = _l._two("x", x), x.dtype, x.device
    dym, xm = _mat("dy", dy, shape, dtype, device), _mat("x", x, shape, dtype, device)
    m, r = _vec("mean", mean, shape[:1], torch.float32, device), _vec("rstd", rstd, shape[:1], torch.float32, device)
    w = _vec("weight", weight, shape[1:], dtype, device)
    dx = x.new_empty(shape) if "x" in need else None
    dw, db = (x.new_empty(shape[1:]) if name in need else None for name in ("weight", "bias"))
    held, p, size = _l._work(L.alpa_norm_backward_work(d, *shape), device)
    binding._check(L.alpa_norm_backward(d, *shape, dym, xm, m, r, w, _l._new(dx), _ptr(dw), _ptr(db), p, size, s))
    return dx, dw, db
