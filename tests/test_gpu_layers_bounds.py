"""Where the layer operators write: through the C ABI, results as parts of buffers whose other bytes are looked at afterwards (bounds of
results: tests/layer_cases.py).  All launches are in bounds by their own checks; nothing here is meant to fault."""
import pytest
import torch

from paper_2201_12023_amd import layers as L
from tests import layer_cases as C

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [BF16, F16, F32]
MARK, MARGIN = 0x5A, 4096


class Guarded:
    """A [rows, n] result, rows `ld` elements apart, `shift` elements behind an aligned address, in a buffer of marked bytes."""

    def __init__(self, rows, n, dtype, pad=0, shift=0):
        es, ld = dtype.itemsize, n + pad
        self.buffer = torch.full((2 * MARGIN + (shift + rows * ld) * es,), MARK, dtype=torch.uint8, device="cuda")
        first = MARGIN // es + shift
        self.view = self.buffer[:self.buffer.numel() // es * es].view(dtype).as_strided((rows, n), (ld, 1), first)
        self.mat = L.alpa_mat_t(self.view.data_ptr(), ld)

    def result(self):
        """What was written; all other bytes are as they were."""
        got = self.view.clone()
        self.view.view(torch.int16 if self.view.element_size() == 2 else torch.int32).fill_(0x5A5A if self.view.element_size() == 2 else 0x5A5A5A5A)
        assert bool((self.buffer == MARK).all())
        return got


class Work:
    """Exactly the work memory that a call asks for, with marks on both sides."""

    def __init__(self, need):
        self.need, self.buffer = need, torch.full((2 * MARGIN + need,), MARK, dtype=torch.uint8, device="cuda")
        self.args = (self.buffer.data_ptr() + MARGIN if need else None, need)

    def check(self):
        assert bool((self.buffer[:MARGIN] == MARK).all()) and bool((self.buffer[MARGIN + self.need:] == MARK).all())


def mat(t):
    return L.alpa_mat_t(t.data_ptr(), t.stride(-2))


NONE = L.alpa_mat_t(None, 0)
DTYPE = {F32: 0, F16: 1, BF16: 2}
stream = lambda: torch.cuda.current_stream().cuda_stream
ENDS = [[3, 40, 40, 120, 129], [0, 0, 0, 0, 0], [0, 1, 2, 130, 131]]
NONSENSE = [[-5, 10, 1000, 20, 7], [40, 30, 20, 10, 0], [2 ** 31 - 1] * 5, [-2 ** 31] * 5, [100, 131, 0, 131, 0], [0, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 131]]


# small and ragged; sizes for which the large tile is taken where results are aligned, and another where not (tests/test_layers_host_side.py)
@pytest.mark.parametrize("pad, shift", [(0, 0), (8, 8), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("rows, n_in, n_out", [(131, 200, 152), (33, 1001, 45), (9000, 5128, 5128)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_dense_layers(dtype, rows, n_in, n_out, pad, shift):
    g, lib, d = C.gen(71), L.load(), DTYPE[dtype]
    x, w, b = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, n_out, n_in, scale=n_in ** -0.5), C.normal(g, dtype, n_out)
    r, dy, z = (C.normal(g, dtype, rows, n_out) for _ in range(3))
    for act in (0, 2, 3):
        y, kept = Guarded(rows, n_out, dtype, pad, shift), Guarded(rows, n_out, dtype, pad, shift)
        work = Work(lib.alpa_linear_forward_work(d, rows, n_in, n_out, mat(x), mat(w)))
        assert lib.alpa_linear_forward(d, act, rows, n_in, n_out, mat(x), mat(w), b.data_ptr(), mat(r), y.mat, kept.mat, *work.args, stream()) == 0
        ry, ey, rz, ez = C.forward(x, w, b, r, act)
        C.within("y", y.result(), ry, ey)
        C.within("z", kept.result(), rz, ez)
        work.check()
        dx, dw, db = Guarded(rows, n_in, dtype, pad, shift), Guarded(n_out, n_in, dtype, pad, shift), Guarded(1, n_out, dtype, 0, shift)
        work = Work(lib.alpa_linear_backward_work(d, act, rows, n_in, n_out, mat(dy), mat(x), mat(w)))
        assert lib.alpa_linear_backward(d, act, rows, n_in, n_out, mat(dy), mat(z) if act else NONE, mat(x), mat(w), dx.mat, dw.mat, db.mat.p, *work.args,
                                        stream()) == 0
        ref = C.backward(dy, z, x, w, act)
        for name, got in (("dx", dx.result()), ("dw", dw.result()), ("dbias", db.result()[0])):
            C.within(name, got, *ref[name])
        work.check()


@pytest.mark.parametrize("pad, shift", [(0, 0), (8, 8), (3, 1)])
@pytest.mark.parametrize("rows, n_in, n_out, grow", [(131, 200, 152, 1), (131, 33, 45, 1), (131 * 96, 2568, 3592, 96)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_expert_layers(dtype, rows, n_in, n_out, grow, pad, shift):
    """Offsets that are right, with empty groups and rows of no expert, and offsets that make no sense, with which results are
    unspecified and all writes stay inside."""
    g, lib, d, E = C.gen(72), L.load(), DTYPE[dtype], 4
    x, w, b = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, E, n_out, n_in, scale=n_in ** -0.5), C.normal(g, dtype, E, n_out)
    r, dy, z = (C.normal(g, dtype, rows, n_out) for _ in range(3))
    for act in (0, 3):
        for ends in ENDS + NONSENSE:
            right = ends in ENDS
            ends = [v * grow if 0 <= v <= 1000 else v for v in ends]
            off = torch.tensor(ends, dtype=torch.int32, device="cuda")
            y, kept = Guarded(rows, n_out, dtype, pad, shift), Guarded(rows, n_out, dtype, pad, shift)
            work = Work(lib.alpa_experts_forward_work(d, rows, E, n_in, n_out, mat(x), mat(w)))
            assert lib.alpa_experts_forward(d, act, rows, E, n_in, n_out, off.data_ptr(), mat(x), mat(w), b.data_ptr(), mat(r), y.mat, kept.mat, *work.args,
                                            stream()) == 0
            y, kept = y.result(), kept.result()
            work.check()
            dx, dw, db = Guarded(rows, n_in, dtype, pad, shift), Guarded(E * n_out, n_in, dtype, pad, shift), Guarded(1, E * n_out, dtype, 0, shift)
            work = Work(lib.alpa_experts_backward_work(d, act, rows, E, n_in, n_out, mat(dy), mat(x), mat(w)))
            assert lib.alpa_experts_backward(d, act, rows, E, n_in, n_out, off.data_ptr(), mat(dy), mat(z) if act else NONE, mat(x), mat(w), dx.mat, dw.mat,
                                             db.mat.p, *work.args, stream()) == 0
            dx, dw, db = dx.result(), dw.result().view(E, n_out, n_in), db.result().view(E, n_out)
            work.check()
            if not right:
                continue
            for t in (y, kept, dx):
                assert not bool(t[:ends[0]].any()) and not bool(t[ends[-1]:].any())
            for e in range(E):
                p = slice(ends[e], ends[e + 1])
                if ends[e] == ends[e + 1]:
                    assert not bool(dw[e].any()) and not bool(db[e].any())
                    continue
                ry, ey, rz, ez = C.forward(x[p], w[e], b[e], r[p], act)
                C.within("y", y[p], ry, ey)
                C.within("z", kept[p], rz, ez)
                ref = C.backward(dy[p], z[p], x[p], w[e], act)
                for name, got in (("dx", dx[p]), ("dw", dw[e]), ("dbias", db[e])):
                    C.within(name, got, *ref[name])


@pytest.mark.parametrize("pad, shift", [(0, 0), (8, 8), (3, 1)])
@pytest.mark.parametrize("rows, n_in, words", [(131, 200, 1000), (70, 33, 77), (1, 8, 1), (20000, 40, 14001), (3001, 1032, 5000)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_loss_over_a_vocabulary(dtype, rows, n_in, words, pad, shift):
    g, lib, d = C.gen(73), L.load(), DTYPE[dtype]
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, words, n_in, scale=n_in ** -0.5)
    t = torch.randint(-words // 10 - 1, words, (rows,), device="cuda", generator=g)
    dloss = torch.rand(rows, device="cuda", generator=g) + 0.5
    loss, lse = Guarded(1, rows, F32, 0, shift), Guarded(1, rows, F32, 0, shift)
    work = Work(lib.alpa_vocab_loss_forward_work(d, rows, n_in, words, mat(x), mat(w)))
    assert lib.alpa_vocab_loss_forward(d, rows, n_in, words, mat(x), mat(w), t.data_ptr(), loss.mat.p, lse.mat.p, *work.args, stream()) == 0
    loss, lse = loss.result()[0], lse.result()[0]
    work.check()
    dx, dw = Guarded(rows, n_in, dtype, pad, shift), Guarded(words, n_in, dtype, pad, shift)
    work = Work(lib.alpa_vocab_loss_backward_work(d, rows, n_in, words, mat(x), mat(w)))
    assert lib.alpa_vocab_loss_backward(d, rows, n_in, words, dloss.data_ptr(), mat(x), mat(w), t.data_ptr(), lse.data_ptr(), dx.mat, dw.mat, *work.args,
                                        stream()) == 0
    ref = C.vocab(x, w, t, dloss)
    for name, got in (("loss", loss), ("lse", lse), ("dx", dx.result()), ("dw", dw.result())):
        C.within(name, got, *ref[name])
    work.check()
