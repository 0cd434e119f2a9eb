"""CPU-side checks of the layer operators' C ABI: exported symbols, and refusals before a device is touched."""
import ctypes
import os
import re

from paper_2201_12023_amd import layers as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "alpa_layers.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(alpa_[a-z_]+)\s*\(", text))
    assert names == set(L.SYMBOLS)
    lib = L.load()
    for n in names:
        assert hasattr(lib, n), n


def M(p, ld):
    return L.alpa_mat_t(p, ld)


P = 1 << 20          # an address that is never followed: every call here is refused


def linear(dtype=2, act=0, rows=4, n_in=8, n_out=6, x=M(P, 8), w=M(P, 8), bias=None, r=M(None, 0), y=M(P, 6), z=M(None, 0), work=None, n=0):
    return L.load().alpa_linear_forward(dtype, act, rows, n_in, n_out, x, w, bias, r, y, z, work, n, None)


def backward(dtype=2, act=3, rows=4, n_in=8, n_out=6, dy=M(P, 6), z=M(P, 6), x=M(P, 8), w=M(P, 8), dx=M(P, 8), dw=M(P, 8), db=None, work=None, n=0):
    return L.load().alpa_linear_backward(dtype, act, rows, n_in, n_out, dy, z, x, w, dx, dw, db, work, n, None)


def test_products_refuse_bad_arguments():
    assert linear(dtype=3) == -1 and linear(dtype=-1) == -1
    assert linear(act=5) == -1 and linear(act=-1) == -1
    assert linear(rows=-1) == -1 and linear(rows=L.MAX_ROWS + 1) == -1
    assert linear(n_in=0) == -1 and linear(n_out=0) == -1
    assert linear(n_in=L.MAX_WIDTH + 1, x=M(P, L.MAX_WIDTH + 1), w=M(P, L.MAX_WIDTH + 1)) == -1
    assert linear(x=M(None, 8)) == -1 and linear(w=M(None, 8)) == -1 and linear(y=M(None, 6)) == -1
    assert linear(x=M(P, 7)) == -1 and linear(x=M(P, (1 << 21) + 1)) == -1 and linear(z=M(P, 5)) == -1
    assert linear(x=M(P + 1, 8)) == -1 and linear(bias=P + 1) == -1
    assert b"stride" in L.load().alpa_dp_last_error() or b"aligned" in L.load().alpa_dp_last_error()
    assert linear(rows=0, x=M(None, 0), y=M(None, 0)) == 0          # nothing to do
    # a product that is split needs work memory
    need = L.load().alpa_linear_forward_work(2, 4, 8192, 64, M(P, 8192), M(P, 8192))
    assert need > 0
    wide = dict(n_in=8192, n_out=64, x=M(P, 8192), w=M(P, 8192), y=M(P, 64))
    assert linear(**wide) == -1 and linear(**wide, work=P, n=need - 1) == -1 and linear(**wide, work=P + 64, n=need) == -1
    assert backward() == -1                                           # dz needs work memory
    assert L.load().alpa_linear_backward_work(2, 3, 4, 8, 6, M(P, 6), M(P, 8), M(P, 8)) > 0
    big = dict(work=P, n=1 << 20)
    assert backward(z=M(None, 0), **big) == -1 and backward(x=M(None, 0), **big) == -1 and backward(w=M(None, 0), **big) == -1
    assert backward(dy=M(None, 0), **big) == -1 and backward(dw=M(P, 7), **big) == -1 and backward(db=P + 1, **big) == -1


def test_experts_and_loss_refuse_bad_arguments():
    lib = L.load()

    def experts(E=2, off=P):
        return lib.alpa_experts_forward(2, 0, 4, E, 8, 6, off, M(P, 8), M(P, 8), None, M(None, 0), M(P, 6), M(None, 0), None, 0, None)

    assert experts(E=0) == -1 and experts(E=L.MAX_EXPERTS + 1) == -1 and experts(off=None) == -1 and experts(off=P + 2) == -1
    assert lib.alpa_experts_backward(2, 0, 4, 0, 8, 6, P, M(P, 6), M(None, 0), M(P, 8), M(P, 8), M(P, 8), M(P, 8), None, P, 1 << 20, None) == -1
    need = lib.alpa_vocab_loss_forward_work(2, 4, 8, 100, M(P, 8), M(P, 8))
    assert need > 0

    def loss(rows=4, words=100, t=P, out=P, work=P, n=need):
        return lib.alpa_vocab_loss_forward(2, rows, 8, words, M(P, 8), M(P, 8), t, out, P, work, n, None)

    assert loss(words=0) == -1 and loss(words=L.MAX_WORDS + 1) == -1 and loss(t=None) == -1 and loss(out=None) == -1
    assert loss(t=P + 4) == -1 and loss(n=need - 1) == -1 and loss(work=None) == -1 and loss(rows=-3) == -1
    need = lib.alpa_vocab_loss_backward_work(2, 4, 8, 100, M(P, 8), M(P, 8))
    args = lambda dloss, n: (2, 4, 8, 100, dloss, M(P, 8), M(P, 8), P, P, M(P, 8), M(P, 8), P, n, None)
    assert lib.alpa_vocab_loss_backward(*args(None, need)) == -1 and lib.alpa_vocab_loss_backward(*args(P, need - 1)) == -1


def test_work_of_refused_sizes_is_none():
    lib, m = L.load(), M(P, 8)
    assert lib.alpa_linear_forward_work(9, 4, 8, 8, m, m) == 0 and lib.alpa_linear_backward_work(2, 3, -1, 8, 8, m, m, m) == 0
    assert lib.alpa_vocab_loss_backward_work(2, 4, 0, 8, m, m) == 0 and lib.alpa_experts_backward_work(2, 3, 4, 0, 8, 8, m, m, m) == 0


def test_work_holds_copies_of_unaligned_operands():
    lib = L.load()
    work = lambda x, w, n_in=4096: lib.alpa_linear_forward_work(2, 4096, n_in, 8192, x, w)
    assert work(M(P, 4096), M(P, 4096)) == 0
    assert work(M(P + 2, 4096), M(P, 4096)) == work(M(P, 4097), M(P, 4096)) == 4096 * 4096 * 2
    assert work(M(P, 4096), M(P, 4100)) == 8192 * 4096 * 2
    assert work(M(P, 4104), M(P, 4096 + 8)) == 0
    assert work(M(P, 4095), M(P, 4095), n_in=4095) == (4096 + 8192) * 4096 * 2
