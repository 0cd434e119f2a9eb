"""The layer operators on the device where types and sizes end (bounds: tests/layer_cases.py)."""
import pytest
import torch

from paper_2201_12023_amd import layers as L
from tests import layer_cases as C

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def gradients(dy, z, x, w, kind):
    """layer_cases.backward for a dz that keeps the bits of a float16 whatever dy's size: it is multiplied by a power of two that
    brings the largest |dy| to 2^13 at least, so a dz is off by U relative and TINY 2^-13 of that largest |dy|."""
    t, rows, n_out = dy.dtype, dy.shape[0], dy.shape[1]
    dy, x, w = dy.to(C.D), x.to(C.D), w.to(C.D)
    dz = dy * C.act(z.to(C.D), kind)[1]
    exact_off = (C.ACT_ERR * 2 + 2 * C.STEP) * dy.abs()
    off = exact_off + C.U[t] * (dz.abs() + exact_off) + C.TINY[t] * 2.0 ** -13 * dy.abs().max()
    out = {}
    for name, a, ao, b, n in (("dx", dz, off, w, n_out), ("dw", dz.t(), off.t(), x, rows)):
        v = a @ b
        e = (ao + (n + 1) * C.STEP * (a.abs() + ao)) @ b.abs()
        out[name] = (v, e + C.U[t] * (v.abs() + e) + C.TINY[t])
    return out


# a dy of 6e4 times a slope of 1.13 is no float16, a dy of 1e-6 has four bits left as one
@pytest.mark.parametrize("kind", [2, 3, 4])
@pytest.mark.parametrize("size, other", [(6e4, 1e-3), (1e-6, 64.0)], ids=["large", "small"])
@pytest.mark.parametrize("pad", [0, 4, 3])
def test_float16_keeps_gradients_of_any_size(kind, size, other, pad):
    g = C.gen(41 + pad)
    rows, n_in, n_out = 517, 72, 264
    x, w = C.normal(g, F16, rows, n_in, scale=other), C.normal(g, F16, n_out, n_in, scale=other)
    wide = (torch.randint(0, 2, (rows, n_out + pad), device="cuda", generator=g) * 2 - 1) * (0.9 + 0.1 * torch.rand(rows, n_out + pad, device="cuda",
                                                                                                               generator=g)) * size
    dy = wide.to(F16)[:, :n_out]
    z = torch.rand(rows, n_out, device="cuda", generator=g).mul_(2.0).add_(0.5).to(F16)
    ref = gradients(dy, z, x, w, kind)
    dx, dw, _ = L.alpa_linear_backward(dy, x, w, z=z, act=kind, need=("x", "w"))
    C.within("dx", dx, *ref["dx"])
    C.within("dw", dw, *ref["dw"])
    # rows of no expert say nothing about the others' size
    ends = [5, 200, 200, 500]
    loud, quiet = torch.full_like(dy, 6e4), torch.zeros(rows, dtype=torch.bool, device="cuda")
    quiet[ends[0]:ends[-1]] = True
    mixed = torch.where(quiet[:, None], dy, loud)
    mixed[-1] = float("nan")
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    ws = torch.stack([w, w, -w])
    dx, dw, _ = L.alpa_experts_backward(mixed, x, ws, off, z=z, act=kind, need=("x", "w"))
    for e in (0, 2):
        p = slice(ends[e], ends[e + 1])
        ref = gradients(dy[p], z[p], x[p], ws[e], kind)
        C.within("dx", dx[p], *ref["dx"])
        C.within("dw", dw[e], *ref["dw"])


def test_float16_gradients_of_zeros_and_of_infinities():
    rows, n_in, n_out = 40, 16, 24
    x, w = torch.ones(rows, n_in, dtype=F16, device="cuda"), torch.ones(n_out, n_in, dtype=F16, device="cuda")
    z = torch.ones(rows, n_out, dtype=F16, device="cuda")
    dy = torch.zeros(rows, n_out, dtype=F16, device="cuda")
    dx, dw, db = L.alpa_linear_backward(dy, x, w, z=z, act=3)
    assert not bool(dx.any()) and not bool(dw.any()) and not bool(db.any())
    dy[3, 5] = float("inf")
    dy[7] = 1e-6
    dx, dw, _ = L.alpa_linear_backward(dy, x, w, z=z, act=4)
    assert bool(torch.isinf(dx[3]).all()) and bool(torch.isinf(dw[5]).all())
    ref = gradients(dy[7:8], z[7:8], x[7:8], w, 4)["dx"]
    C.within("dx", dx[7:8], *ref)
    dy[3, 5] = float("nan")
    dx, dw, _ = L.alpa_linear_backward(dy, x, w, z=z, act=4)
    assert bool(torch.isnan(dx[3]).all()) and bool(torch.isnan(dw[5]).all()) and not bool(torch.isnan(dw[4]).any())


def test_loss_of_more_rows_than_a_launch_has_room_for():
    """2^26 rows and some, 64 threads a row: more threads than HIP counts in a grid."""
    g = C.gen(42)
    rows, n_in, words = (1 << 26) + 21, 8, 3
    w = C.normal(g, BF16, words, n_in)
    x = torch.empty(rows, n_in, dtype=BF16, device="cuda")
    x.view(torch.int16).random_(0x3f80, 0x4000, generator=g)                   # (the bits of 1 to 2)
    t = torch.arange(rows, device="cuda") % (words + 1) - 1
    loss, lse = L.alpa_vocab_loss_forward(x, w, t)
    for part in (slice(0, 50000), slice((1 << 25) - 20000, (1 << 25) + 20000), slice(rows - 50000, rows)):
        ref = C.vocab(x[part], w, t[part], None)
        C.within("loss", loss[part], *ref["loss"])
        C.within("lse", lse[part], *ref["lse"])
    assert bool(torch.isfinite(lse).all()) and not bool(loss[::words + 1].any()) and bool((loss >= 0).all())


def test_gradients_of_more_tiles_than_a_launch_has_room_for():
    """300000 weights for each of 4096 experts, in tiles of 128: two launches (tests/test_layers_host_side.py).  An expert has one
    row or none, so its gradient is one product, exact in 32 bits and rounded once."""
    g = C.gen(43)
    rows, experts, n_in = 1500, 4096, 300000
    has = torch.zeros(experts, dtype=torch.bool, device="cuda")
    has[torch.randperm(experts, device="cuda", generator=g)[:rows]] = True
    off = torch.cat([has.new_zeros(1).int(), torch.cumsum(has, 0).int()])
    assert int(off[-1]) == rows
    x, dy = C.normal(g, BF16, rows, n_in), C.normal(g, BF16, rows, 1)
    w = torch.empty(experts, 1, n_in, dtype=BF16, device="cuda")               # (only its shape is used)
    _, dw, _ = L.alpa_experts_backward(dy, x, w, off, need=("w",))
    assert not bool(dw[~has].any())
    for e0, t0 in ((0, 0), (experts // 2, int(off[experts // 2])), (experts - 200, int(off[experts - 200]))):
        mine = torch.nonzero(has[e0:e0 + 200])[:, 0] + e0
        t = torch.arange(t0, t0 + len(mine), device="cuda")
        assert torch.equal(dw[mine, 0], (dy[t].float() * x[t].float()).to(BF16))


@pytest.mark.parametrize("dtype, rows, words, n_in", [(BF16, 131072 + 1000, 1024, 24), (BF16, 131072 + 1000, 2100, 17), (F32, 3 * 65536 - 77, 1024, 24),
                                                      (F32, 3 * 65536 - 77, 2100, 17), (BF16, 131072 + 28, 1000, 16376), (F32, 65536 + 28, 1000, 16376)], ids=str)
def test_vocab_loss_in_blocks_of_rows(dtype, rows, words, n_in):
    """Rows for which a piece of 1024 words takes more than 256 MiB: dw is the sum of two and more blocks."""
    g = C.gen(44)
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, words, n_in, scale=0.3)
    t = torch.randint(-words // 10, words, (rows,), device="cuda", generator=g)
    dloss = torch.rand(rows, device="cuda", generator=g) / rows
    loss, lse = L.alpa_vocab_loss_forward(x, w, t)
    dx, dw = L.alpa_vocab_loss_backward(dloss, x, w, t, lse)
    dws, bound = torch.zeros(words, n_in, dtype=C.D, device="cuda"), torch.zeros(words, n_in, dtype=C.D, device="cuda")
    step = 16384
    for a in range(0, rows, step):
        part = slice(a, a + step)
        ref = C.vocab(x[part], w, t[part], dloss[part])
        C.within("loss", loss[part], *ref["loss"])
        C.within("dx", dx[part], *ref["dx"])
        dws += ref["dw"][0]
        bound += ref["dw"][1] * (rows / step + 1)    # (sums of `rows` terms in place of 16384)
    C.within("dw", dw, dws, bound)
    only, _ = L.alpa_vocab_loss_backward(dloss, x, w, t, lse, need=("x",))
    _, other = L.alpa_vocab_loss_backward(dloss, x, w, t, lse, need=("w",))
    assert torch.equal(only, dx) and torch.equal(other, dw)


def test_float16_gradients_in_a_graph():
    """The scale of dz is found anew in every replay."""
    g = C.gen(45)
    x, w = C.normal(g, F16, 300, 64), C.normal(g, F16, 136, 64)
    dy, z = C.normal(g, F16, 300, 136), C.normal(g, F16, 300, 136)
    step = lambda: L.alpa_linear_backward(dy, x, w, z=z, act=3)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    for factor in (1.0, 2.0 ** -16, 2.0 ** 20, 2.0 ** -7):
        dy.mul_(factor)
        eager = [v.clone() for v in step()]
        for v in recorded:
            v.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, recorded)) and bool(eager[1].any())
