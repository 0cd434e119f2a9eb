"""The layer operators on the device against their definition in 64 bits (bounds: tests/layer_cases.py)."""
import pytest
import torch

from paper_2201_12023_amd import layers as L
from tests import layer_cases as C

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [BF16, F16, F32]


def ids(v):
    return str(v).replace("torch.", "").replace(" ", "")


def slice_of(t, pad, shift):
    """The same values in a wider buffer: rows `pad` elements further apart, the first `shift` elements in."""
    wide = torch.full((t.shape[0], t.shape[1] + pad + shift), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, shift:shift + t.shape[1]] = t
    return wide[:, shift:shift + t.shape[1]]


# rows, in, out: one of each; blocks of a tile and one more or less; below a chunk; many steps (split); many tiles (the large ones)
SIZES = [(1, 1, 1), (1, 64, 64), (2, 8, 16), (3, 33, 5), (16, 96, 48), (17, 256, 200), (64, 2048, 100), (65, 100, 257), (128, 128, 128), (129, 72, 136),
         (300, 520, 264), (5, 8200, 72), (48, 4096, 96), (70, 1999, 130), (4100, 72, 4104)]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows, n_in, n_out", SIZES)
def test_linear_forward_and_backward(dtype, rows, n_in, n_out):
    g = C.gen(rows * 7 + n_in + n_out)
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, n_out, n_in, scale=n_in ** -0.5)
    b, r, dy = C.normal(g, dtype, n_out), C.normal(g, dtype, rows, n_out), C.normal(g, dtype, rows, n_out)
    for kind in (0, 3) if rows > 1000 else range(5):
        y, z = L.alpa_linear_forward(x, w, bias=b, residual=r, act=kind, keep_z=True)
        ry, ey, rz, ez = C.forward(x, w, b, r, kind)
        C.within("y", y, ry, ey)
        C.within("z", z, rz, ez)
        dx, dw, db = L.alpa_linear_backward(dy, x, w, z=z if kind else None, act=kind)
        ref = C.backward(dy, z, x, w, kind)
        for name, got in (("dx", dx), ("dw", dw), ("dbias", db)):
            C.within(name, got, *ref[name])
    y = L.alpa_linear_forward(x, w)
    C.within("y", y, *C.forward(x, w, None, None, 0)[:2])


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("pad, shift", [(8, 0), (8, 8), (3, 0), (0, 1), (5, 3)])
def test_rows_of_wider_buffers(dtype, pad, shift):
    g = C.gen(pad * 10 + shift)
    rows, n_in, n_out = 131, 200, 152
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, n_out, n_in, scale=n_in ** -0.5)
    r, z, dy = (C.normal(g, dtype, rows, n_out) for _ in range(3))
    xs, ws, rs, zs, dys = (slice_of(t, pad, shift) for t in (x, w, r, z, dy))
    C.within("y", L.alpa_linear_forward(xs, ws, residual=rs, act=4), *C.forward(x, w, None, r, 4)[:2])
    ref = C.backward(dy, z, x, w, 4)
    for name, got in zip(("dx", "dw", "dbias"), L.alpa_linear_backward(dys, xs, ws, z=zs, act=4)):
        C.within(name, got, *ref[name])
    off = torch.tensor([0, 131], dtype=torch.int32, device="cuda")
    C.within("y", L.alpa_experts_forward(xs, w[None], off, act=4), *C.forward(x, w, None, None, 4)[:2])
    t = torch.randint(0, n_out, (rows,), device="cuda", generator=g)
    ref = C.vocab(x, w, t, None)
    loss, lse = L.alpa_vocab_loss_forward(xs, ws, t)
    C.within("loss", loss, *ref["loss"])


def test_offsets_beyond_32_bits():
    """Row 1087 of x begins 2.28e9 elements (4.6e9 bytes) behind the first one."""
    rows, n_in, n_out, ld = 1088, 64, 96, (1 << 21)
    g = C.gen(5)
    buffer = torch.empty(rows * ld, dtype=BF16, device="cuda")
    x = buffer.view(rows, ld)[:, :n_in]
    x.copy_(C.normal(g, BF16, rows, n_in))
    w, dy = C.normal(g, BF16, n_out, n_in), C.normal(g, BF16, rows, n_out)
    C.within("y", L.alpa_linear_forward(x, w), *C.forward(x, w, None, None, 0)[:2])
    _, dw, _ = L.alpa_linear_backward(dy, x, w, need=("w",))
    C.within("dw", dw, *C.backward(dy, None, x, w, 0)["dw"])


def test_extreme_values_of_activations():
    inf = float("inf")
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 20.0, -20.0, 100.0, -100.0, 3e4, -3e4, 1e19, -1e19, 3e38, -3e38, inf, -inf], dtype=F32)
    x = v.cuda()[:, None].contiguous()
    one = torch.ones(1, 1, device="cuda")
    for kind in range(5):
        y = L.alpa_linear_forward(x, one, act=kind)[:, 0].cpu()
        ref = C.act(torch.clamp(v.double(), -1e6, 1e6), kind)[0]
        big = v.abs() > 1e6
        ref[big] = v[big].double() if kind == 0 else torch.clamp(v[big].double(), min=0.0)
        both = torch.isinf(ref)
        assert torch.equal(y[both].double(), ref[both]), kind
        assert bool(((y.double() - ref).abs() <= 2.0 ** -20 * ref.abs() + 2.0 ** -30)[~both].all()), (kind, y, ref)
        if kind:
            dx, _, _ = L.alpa_linear_backward(torch.ones_like(x), x, one, z=x, act=kind, need=("x",))
            slope = C.act(torch.clamp(v.double(), -1e3, 1e3), kind)[1]
            assert bool(((dx[:, 0].cpu().double() - slope).abs() <= 2.0 ** -19).all()), (kind, dx, slope)
        nan = torch.full((1, 1), float("nan"), device="cuda")
        assert bool(torch.isnan(L.alpa_linear_forward(nan, one, act=kind)).all())


# sizes of the groups, rows in front of the first one and behind the last one
GROUPS = [([5], 0, 0), ([0, 0, 0], 0, 3), ([1], 0, 0), ([40, 0, 3, 129, 0], 0, 0), ([0, 17, 64, 1], 2, 5), ([0] * 66 + [3, 200, 0, 9], 1, 0), ([2] * 70, 0, 1),
          ([300, 128, 256], 0, 130)]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("n_in, n_out", [(64, 128), (200, 72), (33, 45)])
@pytest.mark.parametrize("counts, lead, tail", GROUPS, ids=[str(i) for i in range(len(GROUPS))])
def test_experts(dtype, n_in, n_out, counts, lead, tail):
    g = C.gen(len(counts) + n_in)
    E, rows = len(counts), lead + sum(counts) + tail
    ends = [lead]
    for n in counts:
        ends.append(ends[-1] + n)
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x, dy, z = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, rows, n_out), C.normal(g, dtype, rows, n_out)
    w, b = C.normal(g, dtype, E, n_out, n_in, scale=n_in ** -0.5), C.normal(g, dtype, E, n_out)
    r = C.normal(g, dtype, rows, n_out)
    outside = torch.ones(rows, dtype=torch.bool, device="cuda")
    outside[lead:lead + sum(counts)] = False
    for t in (x, dy, z, r):
        t[outside] = float("nan")               # what no expert takes is not looked at
    for kind in (0, 3):
        y, kept = L.alpa_experts_forward(x, w, off, bias=b, residual=r, act=kind, keep_z=True)
        plain = L.alpa_experts_forward(x, w, off, act=kind)
        dx, dw, db = L.alpa_experts_backward(dy, x, w, off, z=z if kind else None, act=kind)
        for t in (y, kept, plain, dx):
            assert not bool(t[outside].any())
        for e in range(E):
            p = slice(ends[e], ends[e + 1])
            if counts[e] == 0:
                assert not bool(dw[e].any()) and not bool(db[e].any())
                continue
            ry, ey, rz, ez = C.forward(x[p], w[e], b[e], r[p], kind)
            C.within("y", y[p], ry, ey)
            C.within("z", kept[p], rz, ez)
            C.within("y", plain[p], *C.forward(x[p], w[e], None, None, kind)[:2])
            ref = C.backward(dy[p], z[p], x[p], w[e], kind)
            for name, got in (("dx", dx[p]), ("dw", dw[e]), ("dbias", db[e])):
                C.within(name, got, *ref[name])


def test_experts_in_large_tiles():
    g = C.gen(12)
    counts = [700, 0, 1, 2047, 1300, 48]
    rows, E, n_in, n_out = sum(counts), len(counts), 136, 4096
    ends = [0]
    for n in counts:
        ends.append(ends[-1] + n)
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x, w, dy = C.normal(g, BF16, rows, n_in), C.normal(g, BF16, E, n_out, n_in, scale=0.1), C.normal(g, BF16, rows, n_out)
    y = L.alpa_experts_forward(x, w, off, act=2)
    dx, dw, db = L.alpa_experts_backward(dy, x, w, off)
    for e in range(E):
        p = slice(ends[e], ends[e + 1])
        C.within("y", y[p], *C.forward(x[p], w[e], None, None, 2)[:2])
        ref = C.backward(dy[p], None, x[p], w[e], 0)
        for name, got in (("dx", dx[p]), ("dw", dw[e]), ("dbias", db[e])):
            C.within(name, got, *ref[name])


# two or more of the largest tiles for each workgroup, edges of tiles in rows and columns, a contraction that ends inside a step
@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_tile_after_tile(dtype):
    g = C.gen(31)
    many, few = (5000, 5128, 568), (5000, 568, 5128)
    for rows, n_in, n_out in ((many[0], many[2], many[1]), few, (568, 5128, 5000)):       # y, dx and dw are the large results in turn
        x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, n_out, n_in, scale=n_in ** -0.5)
        z, dy, b = C.normal(g, dtype, rows, n_out), C.normal(g, dtype, rows, n_out), C.normal(g, dtype, n_out)
        for kind in (0, 2, 4):
            y, kept = L.alpa_linear_forward(x, w, bias=b, residual=dy, act=kind, keep_z=True)
            ry, ey, rz, ez = C.forward(x, w, b, dy, kind)
            C.within("y", y, ry, ey)
            C.within("z", kept, rz, ez)
        ref = C.backward(dy, z, x, w, 4)
        for name, got in zip(("dx", "dw", "dbias"), L.alpa_linear_backward(dy, x, w, z=z, act=4)):
            C.within(name, got, *ref[name])


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_results_larger_than_the_caches(dtype):
    """A result of 256 MiB and more, alone and with z, rows and columns that end inside a tile."""
    g = C.gen(35)
    n_out = 8200 if dtype == F32 else 16392
    x, w, b, r = C.normal(g, dtype, 8203, 72), C.normal(g, dtype, n_out, 72, scale=0.1), C.normal(g, dtype, n_out), C.normal(g, dtype, 8203, n_out)
    for kind, keep in ((0, False), (3, True), (2, False)):
        got = L.alpa_linear_forward(x, w, bias=b, residual=None if keep else r, act=kind, keep_z=keep)
        ry, ey, rz, ez = C.forward(x, w, b, None if keep else r, kind)
        C.within("y", got[0] if keep else got, ry, ey)
        if keep:
            C.within("z", got[1], rz, ez)


@pytest.mark.parametrize("bytes_apart", [0, 8, 2])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_slopes_of_few_and_of_many_rows(dtype, bytes_apart):
    """dz with slots of 16 and of 64 rows, read by 16 bytes, by 8 and by elements, dense and ragged."""
    g = C.gen(36)
    pad = 0 if bytes_apart == 0 else max(bytes_apart // dtype.itemsize, 1)
    for rows, n_out in ((331, 520), (8203, 4104)):
        x, w = C.normal(g, dtype, rows, 24), C.normal(g, dtype, n_out, 24, scale=0.2)
        dy, z = C.normal(g, dtype, rows, n_out), C.normal(g, dtype, rows, n_out)
        dys, zs = (slice_of(t, pad, 0) for t in (dy, z))
        ref = C.backward(dy, z, x, w, 2)
        for name, got in zip(("dx", "dw", "dbias"), L.alpa_linear_backward(dys, x, w, z=zs, act=2)):
            C.within(name, got, *ref[name])
        ends = [0, 0, rows // 3, rows // 3 + 17, rows - 5]
        off = torch.tensor(ends, dtype=torch.int32, device="cuda")
        ws = torch.stack([w] * 4)
        dx, dw, db = L.alpa_experts_backward(dys, x, ws, off, z=zs, act=2)
        for e in range(4):
            p = slice(ends[e], ends[e + 1])
            if ends[e] == ends[e + 1]:
                assert not bool(dw[e].any()) and not bool(db[e].any())
                continue
            ref = C.backward(dy[p], z[p], x[p], w, 2)
            for name, got in (("dx", dx[p]), ("dw", dw[e]), ("dbias", db[e])):
                C.within(name, got, *ref[name])


def test_experts_tile_after_tile():
    g = C.gen(32)
    counts = [1700, 0, 3, 2500, 900, 0, 260]
    rows, E, n_in, n_out = sum(counts) + 70, len(counts), 1032, 4104
    ends = [0]
    for n in counts:
        ends.append(ends[-1] + n)
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x, w, dy = C.normal(g, BF16, rows, n_in), C.normal(g, BF16, E, n_out, n_in, scale=0.03), C.normal(g, BF16, rows, n_out)
    z, b = C.normal(g, BF16, rows, n_out), C.normal(g, BF16, E, n_out)
    for t in (x, dy, z):
        t[ends[-1]:] = float("nan")
    wide = torch.randn(E, n_in, n_out, device="cuda", generator=g).mul_(0.03).to(BF16)     # the other way, so that dx is large too
    for act, xx, dd, zz, ww, bb in ((3, x, dy, z, w, b), (0, dy, x, x, wide, None)):
        y, kept = L.alpa_experts_forward(xx, ww, off, bias=bb, act=act, keep_z=True)
        dx, dw, db = L.alpa_experts_backward(dd, xx, ww, off, z=zz if act else None, act=act)
        for t in (y, kept, dx):
            assert not bool(t[ends[-1]:].any())
        for e in range(E):
            p = slice(ends[e], ends[e + 1])
            if counts[e] == 0:
                assert not bool(dw[e].any()) and not bool(db[e].any())
                continue
            ry, ey, rz, ez = C.forward(xx[p], ww[e], None if bb is None else bb[e], None, act)
            C.within("y", y[p], ry, ey)
            C.within("z", kept[p], rz, ez)
            ref = C.backward(dd[p], zz[p], xx[p], ww[e], act)
            for name, got in (("dx", dx[p]), ("dw", dw[e]), ("dbias", db[e])):
                C.within(name, got, *ref[name])


@pytest.mark.parametrize("dtype", [BF16, F16], ids=ids)
def test_vocab_loss_tile_after_tile(dtype):
    g = C.gen(33)
    rows, n_in, words = 3000, 1032, 10504
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, words, n_in, scale=0.05)
    t = torch.randint(0, words, (rows,), device="cuda", generator=g)
    t[::7] = -100
    dloss = torch.rand(rows, device="cuda", generator=g)
    ref = C.vocab(x, w, t, dloss)
    loss, lse = L.alpa_vocab_loss_forward(x, w, t)
    C.within("loss", loss, *ref["loss"])
    dx, dw = L.alpa_vocab_loss_backward(dloss, x, w, t, lse)
    C.within("dx", dx, *ref["dx"])
    C.within("dw", dw, *ref["dw"])


def test_offsets_that_make_no_sense_stay_inside():
    """Results are unspecified, but nothing outside the tensors is touched and the calls end."""
    x, w = torch.ones(50, 64, dtype=BF16, device="cuda"), torch.ones(3, 32, 64, dtype=BF16, device="cuda")
    guard = torch.full((3, 50, 32), 7.0, dtype=BF16, device="cuda")
    for bad in ([-5, 10, 1000, 20], [40, 30, 20, 10], [2 ** 31 - 1] * 4, [-2 ** 31] * 4):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        L.alpa_experts_forward(x, w, off, act=1)
        L.alpa_experts_backward(guard[1], x, w, off, z=guard[1], act=1)
    torch.cuda.synchronize()
    assert bool((guard == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows, n_in, words", [(1, 64, 1), (1, 64, 100), (2, 33, 77), (17, 128, 64), (130, 200, 1000), (129, 96, 5003),
                                              (300, 72, 513)])
def test_vocab_loss(dtype, rows, n_in, words):
    g = C.gen(rows + words)
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, words, n_in, scale=2 * n_in ** -0.5)
    t = torch.randint(0, words, (rows,), device="cuda", generator=g)
    t[torch.rand(rows, device="cuda", generator=g) < 0.2] = -100
    t[0] = words - 1
    dloss = torch.randn(rows, device="cuda", generator=g)
    ref = C.vocab(x, w, t, dloss)
    loss, lse = L.alpa_vocab_loss_forward(x, w, t)
    C.within("loss", loss, *ref["loss"])
    C.within("lse", lse, *ref["lse"])
    dx, dw = L.alpa_vocab_loss_backward(dloss, x, w, t, lse)
    C.within("dx", dx, *ref["dx"])
    C.within("dw", dw, *ref["dw"])
    assert not bool(loss[t < 0].any()) and not bool(dx[t < 0].any())
    only, none = L.alpa_vocab_loss_backward(dloss, x, w, t, lse, need=("x",))
    assert none is None and torch.equal(only, dx)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=ids)
def test_vocab_loss_in_several_pieces(dtype):
    """Rows enough that the gradient of the logits does not fit in one piece."""
    g = C.gen(3)
    rows, n_in, words = 20000, 32, 14001
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, words, n_in, scale=0.3)
    mats = [L.alpa_mat_t(t.data_ptr(), n_in) for t in (x, w)]
    assert L.load().alpa_vocab_loss_backward_work(0 if dtype == F32 else 2, rows, n_in, words, *mats) < rows * words * x.element_size()
    t = torch.randint(0, words, (rows,), device="cuda", generator=g)
    dloss = torch.full((rows,), 1.0 / rows, device="cuda")
    loss, lse = L.alpa_vocab_loss_forward(x, w, t)
    dx, dw = L.alpa_vocab_loss_backward(dloss, x, w, t, lse)
    dws = torch.zeros(words, n_in, dtype=C.D, device="cuda")
    bound = torch.zeros_like(dws)
    for a in range(0, rows, 4000):
        ref = C.vocab(x[a:a + 4000], w, t[a:a + 4000], dloss[a:a + 4000])
        C.within("loss", loss[a:a + 4000], *ref["loss"])
        C.within("dx", dx[a:a + 4000], *ref["dx"])
        dws += ref["dw"][0]
        bound += ref["dw"][1] * 5                # (the sum of 20000 terms in place of 4000)
    C.within("dw", dw, dws, bound)


def test_vocab_loss_of_extreme_logits():
    # one word far above the others, all equal, and overflowing to infinity
    x = torch.tensor([[1.0], [0.0], [1e30]], device="cuda")
    w = torch.tensor([[100.0], [0.0], [-100.0], [1e30]], device="cuda")[:3].contiguous()
    t = torch.tensor([0, 1, 2], device="cuda")
    loss, lse = L.alpa_vocab_loss_forward(x, w, t)
    assert float(loss[0]) == 0.0 and abs(float(loss[1]) - 1.0986123) < 1e-6 and float(loss[2]) == pytest.approx(2e32)
    none = torch.full((3,), -1, device="cuda")
    loss, lse = L.alpa_vocab_loss_forward(x, w, none)
    assert not bool(loss.any())
    dx, dw = L.alpa_vocab_loss_backward(torch.ones(3, device="cuda"), x, w, none, lse)
    assert not bool(dx.any()) and not bool(dw.any())
    loss, lse = L.alpa_vocab_loss_forward(x, w, torch.tensor([0, 3, 1], device="cuda"))      # 3 is no word
    assert bool(torch.isnan(loss[1])) and not bool(torch.isnan(loss[0]))
    zero = torch.zeros(3, device="cuda")
    dx, dw = L.alpa_vocab_loss_backward(zero, x[:2].repeat(2, 1)[:3].contiguous(), w, t, lse)
    assert not bool(dx.any()) and not bool(dw.any())


def test_gradients_against_differences():
    """Central differences of the operators' own forward results in 32 bits; h^2 times the third derivative and 2^-23 / h of the sums stay
    below the tolerance of 2e-3 of the largest gradient."""
    g = C.gen(9)
    rows, n_in, n_out, h = 6, 5, 7, 2.0 ** -6
    x, w, b = C.normal(g, F32, rows, n_in), C.normal(g, F32, n_out, n_in), C.normal(g, F32, n_out)
    dy = C.normal(g, F32, rows, n_out)
    off = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    w2, b2 = torch.stack([w, w.flip(0).contiguous()]), torch.stack([b, -b])
    t = torch.tensor([0, 6, -1, 3, 3, 2], device="cuda")
    dloss = C.normal(g, F32, rows)

    def check(value, tensors, grads):
        for v, grad in zip(tensors, grads):
            flat, diff = v.view(-1), torch.zeros(v.numel(), dtype=C.D)
            for j in range(v.numel()):
                old = flat[j].clone()
                flat[j] = old + h
                up = value()
                flat[j] = old - h
                diff[j] = (up - value()) / (2 * h)
                flat[j] = old
            err = (grad.cpu().double().view(-1) - diff).abs().max()
            assert float(err) <= 2e-3 * float(diff.abs().max()) + 1e-4, err

    for kind in (0, 2, 3, 4):
        y, z = L.alpa_linear_forward(x, w, bias=b, act=kind, keep_z=True)
        check(lambda: float((L.alpa_linear_forward(x, w, bias=b, act=kind).double() * dy).sum()), (x, w, b),
              L.alpa_linear_backward(dy, x, w, z=z, act=kind))
        y, z = L.alpa_experts_forward(x, w2, off, bias=b2, act=kind, keep_z=True)
        check(lambda: float((L.alpa_experts_forward(x, w2, off, bias=b2, act=kind).double() * dy).sum()), (x, w2, b2),
              L.alpa_experts_backward(dy, x, w2, off, z=z, act=kind))
    loss, lse = L.alpa_vocab_loss_forward(x, w, t)
    check(lambda: float((L.alpa_vocab_loss_forward(x, w, t)[0].double() * dloss).sum()), (x, w),
          L.alpa_vocab_loss_backward(dloss, x, w, t, lse))


def test_no_rows():
    x, w, off = torch.empty(0, 16, device="cuda"), torch.ones(8, 16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    dy, t = torch.empty(0, 8, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    assert L.alpa_linear_forward(x, w).shape == (0, 8)
    dx, dw, db = L.alpa_linear_backward(dy, x, w)
    assert dx.shape == (0, 16) and not bool(dw.any()) and not bool(db.any())
    w2 = torch.ones(2, 8, 16, device="cuda")
    assert L.alpa_experts_forward(x, w2, off).shape == (0, 8)
    dx, dw, db = L.alpa_experts_backward(dy, x, w2, off)
    assert dw.shape == (2, 8, 16) and not bool(dw.any()) and not bool(db.any())
    loss, lse = L.alpa_vocab_loss_forward(x, w, t)
    dx, dw = L.alpa_vocab_loss_backward(loss, x, w, t, lse)
    assert loss.shape == (0,) and not bool(dw.any())


def test_same_bits_on_any_stream_and_in_graphs():
    g = C.gen(21)
    rows, n_in, n_out = 70, 1536, 200
    x, w, b = C.normal(g, BF16, rows, n_in), C.normal(g, BF16, n_out, n_in, scale=0.03), C.normal(g, BF16, n_out)
    dy = C.normal(g, BF16, rows, n_out)
    t = torch.randint(0, n_out, (rows,), device="cuda", generator=g)
    off = torch.tensor([0, 30, 30, 65], dtype=torch.int32, device="cuda")
    w3 = torch.stack([w, w, -w]).contiguous()
    dloss = torch.ones(rows, device="cuda")

    def step():
        y, z = L.alpa_linear_forward(x, w, bias=b, act=3, keep_z=True)
        out = [y, z, *L.alpa_linear_backward(dy, x, w, z=z, act=3), L.alpa_experts_forward(x, w3, off, act=4)]
        out += L.alpa_experts_backward(dy, x, w3, off, z=z, act=4)
        loss, lse = L.alpa_vocab_loss_forward(x, w, t)
        return out + [loss, lse, *L.alpa_vocab_loss_backward(dloss, x, w, t, lse)]

    first = [v.clone() for v in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, c) for a, c in zip(first, second))
    y = L.alpa_linear_forward(x, w, bias=b, act=3, stream=side)
    side.synchronize()
    assert torch.equal(y, first[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    for k in range(4):
        x.mul_(-1.0)                             # the program's own work between the replays, and other inputs
        dy.mul_(0.5)
        eager = [v.clone() for v in step()]
        for v in recorded:
            v.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(eager, recorded)), k


def test_refusals():
    x, w = torch.ones(4, 8, device="cuda"), torch.ones(6, 8, device="cuda")
    dy, t = torch.ones(4, 6, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    bad = [
        lambda: L.alpa_linear_forward(x.double(), w.double()),                     # type
        lambda: L.alpa_linear_forward(x, w.half()),
        lambda: L.alpa_linear_forward(x, w.cpu()),
        lambda: L.alpa_linear_forward(x.cpu(), w.cpu()),
        lambda: L.alpa_linear_forward(x[0], w),                                    # shapes
        lambda: L.alpa_linear_forward(x, w[:, :7]),
        lambda: L.alpa_linear_forward(x, w, bias=torch.ones(5, device="cuda")),
        lambda: L.alpa_linear_forward(x, w, residual=x),
        lambda: L.alpa_linear_forward(x.t().contiguous().t(), w),                  # strides
        lambda: L.alpa_linear_forward(x[:1].expand(4, 8), w),
        lambda: L.alpa_linear_forward(x, w, bias=torch.ones(12, device="cuda")[::2]),
        lambda: L.alpa_linear_backward(dy, x, w, need=("dx",)),
        lambda: L.alpa_linear_backward(dy, None, None),
        lambda: L.alpa_experts_forward(x, w, off),                                 # w without experts
        lambda: L.alpa_experts_forward(x, w[None], off.long()),
        lambda: L.alpa_experts_forward(x, torch.ones(2, 6, 8, device="cuda"), off),
        lambda: L.alpa_experts_forward(x, torch.ones(2, 8, 8, device="cuda")[:, :6], torch.zeros(3, dtype=torch.int32, device="cuda")),
        lambda: L.alpa_vocab_loss_forward(x, w, t.int()),
        lambda: L.alpa_vocab_loss_forward(x, w, t[:3]),
        lambda: L.alpa_vocab_loss_backward(torch.ones(4, device="cuda", dtype=torch.float64), x, w, t, torch.ones(4, device="cuda")),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted:", k)
    refused = [
        lambda: L.alpa_linear_forward(x, w, act=5),
        lambda: L.alpa_linear_backward(dy, x, w, act=3),                           # an activation without z
        lambda: L.alpa_linear_backward(dy, None, w, need=("w",)),                  # dw without x
        lambda: L.alpa_linear_backward(dy, x, None, need=("x",)),
    ]
    for k, call in enumerate(refused):
        with pytest.raises(L.binding.AlpaDpError):
            call()
            print("accepted:", k)
