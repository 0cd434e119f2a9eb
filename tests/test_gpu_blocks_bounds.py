"""Where attention, rotary positions and layer norm write: through the C ABI, results as parts of buffers whose other bytes are looked at afterwards, with exactly
the work memory that a call asks for.  All launches are in bounds by their own checks; nothing here is meant to fault."""
import pytest
import torch

from paper_2201_12023_amd import blocks as B
from paper_2201_12023_amd import layers as L
from tests import block_cases as C
from tests.layer_cases import gen, normal
from tests.test_gpu_layers_bounds import DTYPE, MARGIN, MARK, Guarded, Work, mat, stream

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [BF16, F16, F32]
NONSENSE = [[-5, 10, 1000, 20, 7], [40, 30, 20, 10, 0], [2 ** 31 - 1] * 5, [-2 ** 31] * 5, [100, 131, 0, 131, 0], [0, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 131]]


class Heads:
    """A [rows, heads, dim] result with room between heads and between rows, in a buffer of marked bytes; `turned`: heads outside, rows inside."""

    def __init__(self, rows, heads, dim, dtype, pad=0, shift=0, turned=False):
        es = dtype.itemsize
        inner, outer = (rows, heads) if turned else (heads, rows)
        step = dim + pad
        far = inner * step + pad
        self.buffer = torch.full((2 * MARGIN + (shift + outer * far) * es,), MARK, dtype=torch.uint8, device="cuda")
        strides = (step, far, 1) if turned else (far, step, 1)
        self.view = self.buffer[:self.buffer.numel() // es * es].view(dtype).as_strided((rows, heads, dim), strides, MARGIN // es + shift)
        self.heads = B.alpa_heads_t(self.view.data_ptr(), *strides[:2])

    def result(self):
        got = self.view.clone()
        wide = self.view.element_size() == 4
        self.view.view(torch.int32 if wide else torch.int16).fill_(0x5A5A5A5A if wide else 0x5A5A)
        assert bool((self.buffer == MARK).all())
        return got


def heads(t):
    return B.alpa_heads_t(t.data_ptr(), t.stride(0), t.stride(1))


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def how(q, k, off, k_off, causal=1, cap=0.0, slopes=None, prefix=None):
    p = lambda t: None if t is None else t.data_ptr()
    pairs = k_off is not None and k_off.dim() == 2
    return B.alpa_attention_t(DTYPE[q.dtype], 1 if off is None else off.numel() - 1, q.shape[1], k.shape[1], q.shape[2], causal, 2 if pairs else 1, q.shape[2] ** -0.5,
                              cap, q.shape[0], k.shape[0], p(off), p(k_off), p(prefix), p(slopes))


def run(q, k, v, dy, off, k_off, place=lambda *a: Heads(*a), **more):
    """y, lse, dq, dk, dv of the two calls, looked at around"""
    lib, a = B.load(), how(q, k, off, k_off, **more)
    rows, n, dim = q.shape
    y, lse = place(rows, n, dim, q.dtype), Guarded(rows, n, F32)
    work = Work(lib.alpa_attention_forward_work(a, heads(q), heads(k), heads(v)))
    assert lib.alpa_attention_forward(a, heads(q), heads(k), heads(v), y.heads, lse.mat.p, *work.args, stream()) == 0
    work.check()
    got = [y.view.clone(), lse.view.clone()]
    if dy is not None:
        dq, dk, dv = place(rows, n, dim, q.dtype), place(*k.shape, q.dtype), place(*k.shape, q.dtype)
        ops = [heads(t) for t in (dy, q, k, v, y.view)]
        work = Work(lib.alpa_attention_backward_work(a, *ops))
        assert lib.alpa_attention_backward(a, *ops, lse.mat.p, dq.heads, dk.heads, dv.heads, *work.args, stream()) == 0
        work.check()
        got += [dq.result(), dk.result(), dv.result()]
    y.result(), lse.result()
    return got


@pytest.mark.parametrize("pad, shift, turned", [(0, 0, False), (8, 8, False), (3, 0, False), (0, 1, False), (8, 0, True), (5, 3, True)])
@pytest.mark.parametrize("dtype, dim", [(BF16, 64), (BF16, 75), (F16, 128), (F32, 36), (BF16, 256), (F32, 200)])
def test_attention(dtype, dim, pad, shift, turned):
    """Operands and results with all distances between heads and rows: the same as from tensors without any."""
    g = gen(dim + pad)
    rows, k_rows, n, kv = 150, 170, 4, 2
    off, k_off = ints([2, 40, 40, 140]), ints([0, 60, 61, 165])

    def placed(*shape):
        t = Heads(*shape, dtype, pad, shift, turned).view
        t.copy_(normal(g, dtype, *shape))
        return t
    q, k, v, dy = placed(rows, n, dim), placed(k_rows, kv, dim), placed(k_rows, kv, dim), placed(rows, n, dim)
    got = run(q, k, v, dy, off, k_off, lambda *a: Heads(*a, pad, shift, turned))
    ref = run(*(t.contiguous() for t in (q, k, v, dy)), off, k_off)
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    exact = C.attention(q, k, v, dy, off, k_off, causal=True)
    for name, t in zip(("y", "lse", "dq", "dk", "dv"), got):
        C.within(name, t, exact[name])


@pytest.mark.parametrize("ends", NONSENSE, ids=str)
@pytest.mark.parametrize("which", ["rows", "keys", "both"])
@pytest.mark.parametrize("dim", [64, 75])
def test_offsets_that_are_none(ends, which, dim):
    """Any offsets: unspecified results, nothing written or read elsewhere."""
    g = gen(1)
    q, k, v, dy = (normal(g, BF16, 131, n, dim) for n in (6, 2, 2, 6))
    good = ints([0, 30, 60, 100, 131])
    off, k_off = (ints(ends) if which != "keys" else good), (ints(ends) if which != "rows" else good)
    run(q, k, v, dy, off, k_off, prefix=ints([-7, 2 ** 31 - 1, 50, -2 ** 31]))
    run(q, k, v, None, off, ints([[a, b] for a, b in zip(ends, ends[::-1])][:4]))


@pytest.mark.parametrize("rows, k_rows", [(0, 5), (5, 0), (0, 0)])
def test_attention_of_nothing(rows, k_rows):
    g = gen(2)
    q, k, v, dy = (normal(g, BF16, r, n, 64) for r, n in ((rows, 4), (k_rows, 2), (k_rows, 2), (rows, 4)))
    y, lse = B.alpa_attention_forward(q, k, v, causal=True, keep_lse=True)
    assert bool((y == 0).all()) and bool((lse == -float("inf")).all())
    for t in B.alpa_attention_backward(dy, q, k, v, y, lse, causal=True):
        assert bool((t == 0).all())


@pytest.mark.parametrize("pad, shift, turned", [(0, 0, False), (4, 0, False), (3, 1, False), (8, 0, True)])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, n, dim, rot", [(33, 5, 64, 64), (7, 3, 80, 20), (5, 2, 75, 30)])
def test_rotary(dtype, rows, n, dim, rot, interleaved, pad, shift, turned):
    g, lib = gen(3), B.load()
    x, out = Heads(rows, n, dim, dtype, pad, shift, turned), Heads(rows, n, dim, dtype, pad, shift, turned)
    x.view.copy_(normal(g, dtype, rows, n, dim))
    pos, f = torch.arange(rows, device="cuda") * 1000003, B.alpa_rotary_frequencies(rot)
    ref = C.rotary(x.view, pos, f, bool(interleaved), 1.0)
    args = (DTYPE[dtype], rows, n, dim, rot, interleaved, 1.0, pos.data_ptr(), f.data_ptr())
    assert lib.alpa_rotary_forward(*args, x.heads, out.heads, stream()) == 0
    C.within("y", out.result(), ref)
    assert lib.alpa_rotary_forward(*args, x.heads, x.heads, stream()) == 0          # in place
    C.within("in place", x.result(), ref)


@pytest.mark.parametrize("pad, shift", [(0, 0), (8, 8), (3, 1)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, n", [(33, 1000), (5, 4096), (3, 20000), (2500, 72)])
def test_norm(dtype, rows, n, pad, shift):
    g, lib, d = gen(4), B.load(), DTYPE[dtype]
    x, dy = (Guarded(rows, n, dtype, pad, shift).view for _ in range(2))
    x.copy_(normal(g, dtype, rows, n) + 0.5)
    dy.copy_(normal(g, dtype, rows, n))
    vec = lambda t: torch.cat([torch.zeros(shift, dtype=dtype, device="cuda"), t])[shift:]
    w, b = vec(normal(g, dtype, n)), vec(normal(g, dtype, n))
    ref = C.norm(x, w, b, 1e-5, dy)
    y, dx = Guarded(rows, n, dtype, pad, shift), Guarded(rows, n, dtype, pad, shift)
    mean, rstd, dw, db = Guarded(1, rows, F32), Guarded(1, rows, F32), Guarded(1, n, dtype, 0, shift), Guarded(1, n, dtype, 0, shift)
    assert lib.alpa_norm_forward(d, rows, n, 1e-5, mat(x), w.data_ptr(), b.data_ptr(), y.mat, mean.mat.p, rstd.mat.p, stream()) == 0
    work = Work(lib.alpa_norm_backward_work(d, rows, n))
    assert lib.alpa_norm_backward(d, rows, n, mat(dy), mat(x), mean.mat.p, rstd.mat.p, w.data_ptr(), dx.mat, dw.mat.p, db.mat.p, *work.args, stream()) == 0
    work.check()
    for name, t in (("y", y), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dweight", dw), ("dbias", db)):
        got = t.result()
        C.within(name, got[0] if got.shape[0] == 1 and rows > 1 else got, ref[name])
