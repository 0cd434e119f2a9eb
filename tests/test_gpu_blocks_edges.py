"""Attention, rotary positions and layer norm at the edges of their types and sizes, on streams, in graphs, and as nodes of torch's graph."""
import math

import pytest
import torch

from paper_2201_12023_amd import blocks as B
from tests import block_cases as C
from tests.layer_cases import D, gen, normal

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [BF16, F16, F32]


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def both(q, k, v, dy, **how):
    y, lse = B.alpa_attention_forward(q, k, v, keep_lse=True, **how)
    return y, lse, *B.alpa_attention_backward(dy, q, k, v, y, lse, **how)


# one: within a range of its own, mixed: rows, and keys, of a sequence many orders of magnitude apart
@pytest.mark.parametrize("size", [6e4, 1.0, 1e-3, 3e-6, "mixed"])
@pytest.mark.parametrize("rows", [100, 900])
def test_gradients_of_all_sizes_in_float16(size, rows):
    """dR neither overflows nor loses the bits of small gradients: within block_cases' bounds, which go down with the largest |dR| of a row or key and only at the end have
    float16's smallest step.  (A bound relative to a row's result alone does not hold: the first row sees one key, its dP - delta is zero, and what the kernel has there
    is the rounding of two sums of 64 products of dy and v, up to 66 * 2^-23 * sum |dy v|, and of delta's y, 2^-11 |dy| |y|, which the bounds count.)"""
    g = gen(21)
    q, k, v, dy = normal(g, F16, rows, 4, 64), normal(g, F16, rows, 2, 64), normal(g, F16, rows, 2, 64, scale=0.05 if size == 6e4 else 1.0), normal(g, F16, rows, 4, 64).float()
    top = dy.abs().max()
    if size == "mixed":
        # (values of 1e-5 have bits of 2^-24 left: what they are after rounding is what counts)
        dy = dy * (10.0 ** (-5 * torch.rand(rows, 1, 1, device="cuda", generator=g)))
    else:
        dy = dy / top * size
    dy = dy.to(F16)
    _, _, dq, dk, dv = both(q, k, v, dy, causal=True)
    ref = C.attention(q, k, v, dy, causal=True)
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        value, bound = ref[name]
        fits = (value.abs() + bound).amax((1, 2)) < 65504
        assert bool(fits.any())
        C.within(name, got[fits], (value[fits], bound[fits]))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_scores_far_apart(dtype):
    """Scores of a thousand and more: one key takes all the weight; exponentials that are far below vanish without a NaN."""
    g = gen(22)
    q, k = normal(g, dtype, 90, 2, 64, scale=12.0), normal(g, dtype, 90, 2, 64, scale=12.0)
    v, dy = normal(g, dtype, 90, 2, 64), normal(g, dtype, 90, 2, 64)
    ref = C.attention(q, k, v, dy, causal=True)
    for name, got in zip(("y", "lse", "dq", "dk", "dv"), both(q, k, v, dy, causal=True)):
        assert bool(torch.isfinite(got.float()).all()), name
        C.within(name, got, ref[name])
    # growing along the keys, so that the reference is raised again and again
    ramp = torch.linspace(-40, 40, 700, device="cuda")
    k = torch.zeros(700, 1, 64, device="cuda", dtype=dtype)
    k[:, 0, 0] = ramp.to(dtype)
    q = torch.zeros(5, 1, 64, device="cuda", dtype=dtype)
    q[:, 0, 0] = torch.tensor([1.0, -1.0, 8.0, -8.0, 0.0]).to(dtype)
    v = normal(g, dtype, 700, 1, 64)
    ref = C.attention(q, k, v, scale=1.0)
    y, lse = B.alpa_attention_forward(q, k, v, scale=1.0, keep_lse=True)
    C.within("y", y, ref["y"])
    C.within("lse", lse, ref["lse"])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=str)
def test_infinities_and_numbers_that_are_none(dtype):
    """They stay within their sequence and kv head, and a score that is infinite and one that is no number give no numbers."""
    g = gen(23)
    off = ints(0, 40, 80, 120)
    q, k, v, dy = normal(g, dtype, 130, 4, 64), normal(g, dtype, 130, 2, 64), normal(g, dtype, 130, 2, 64), normal(g, dtype, 130, 4, 64)
    clean = both(q, k, v, dy, offsets=off, causal=True)
    for t, value in ((q, math.nan), (k, math.inf), (v, math.nan), (dy, -math.inf)):
        was = t[50, 0].clone()
        t[50, 0] = value
        t[125:] = value                                   # (rows and keys of no sequence are not read)
        got = both(q, k, v, dy, offsets=off, causal=True)
        t[50, 0] = was
        for a, b in zip(got, clean):
            kept = torch.ones_like(b, dtype=torch.bool)
            kept[40:80, :b.shape[1] // 2] = False         # the query heads of kv head 0
            assert torch.equal(a[kept], b[kept])
        assert not bool(torch.isfinite(got[0][50 if t is not dy else 0:80, 0].float()).all()) or t is dy
        t[125:] = 0.0
    # rows behind an infinite score: no number, as from the definition
    q1, k1 = torch.ones(1, 1, 64, device="cuda", dtype=dtype), torch.ones(3, 1, 64, device="cuda", dtype=dtype)
    k1[1] = math.inf
    y, lse = B.alpa_attention_forward(q1, k1, torch.ones(3, 1, 64, device="cuda", dtype=dtype), keep_lse=True)
    assert bool(torch.isnan(y.float()).all())


def test_a_cache_longer_than_32_bits_reach():
    """Keys whose elements lie behind 2^32 bytes and 2^31 elements: the last sequence's, against the same keys alone."""
    g, dim, kv = gen(24), 128, 8
    rows = (1 << 31) // (dim * kv) + 4096
    k = torch.zeros(rows, kv, dim, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    n = 3000
    k[-n:], v[-n:] = normal(g, BF16, n, kv, dim), normal(g, BF16, n, kv, dim)
    q = normal(g, BF16, 2, 16, dim)
    pairs = ints([5, 400], [rows - n, rows])
    y = B.alpa_attention_forward(q, k, v, ints(0, 1, 2), pairs, causal=True)
    alone = B.alpa_attention_forward(q[1:], k[-n:].clone(), v[-n:].clone(), causal=True)
    assert float((y[1].float() - alone[0].float()).abs().max()) <= 2 * 2.0 ** -8 * float(alone.float().abs().max())       # (other parts of the keys)
    assert bool((y[0] == 0).all())


@pytest.mark.parametrize("apart", [1 << 21, (1 << 21) + 8])
def test_rows_far_apart(apart):
    """Rows 2^22 bytes apart, the most that is read in place, and further: the same as from rows behind one another."""
    g, room = gen(31), torch.empty(300 * apart, dtype=BF16, device="cuda")
    tensors = [normal(g, BF16, 300, n, 128) for n in (4, 2, 2, 4)]
    ref = both(*tensors, causal=True)
    far = [room.as_strided(t.shape, (apart, 128, 1), k * 1024) for k, t in enumerate(tensors)]
    for t, f in zip(tensors, far):
        f.copy_(t)
    for a, b in zip(both(*far, causal=True), ref):
        assert torch.equal(a, b)
    # heads far apart, rows beside one another
    far = [room.as_strided(t.shape, (512, apart * 40, 1), k * 128) for k, t in enumerate(tensors)]
    for t, f in zip(tensors, far):
        f.copy_(t)
    for a, b in zip(both(*far, causal=True), ref):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_the_same_bits_twice(dtype):
    g = gen(25)
    off = ints(0, 700, 1500)
    q, k, v, dy = normal(g, dtype, 1500, 8, 64), normal(g, dtype, 1500, 2, 64), normal(g, dtype, 1500, 2, 64), normal(g, dtype, 1500, 8, 64)
    first = both(q, k, v, dy, offsets=off, causal=True, cap=20.0)
    junk = torch.full((1 << 28,), 0x7F, dtype=torch.uint8, device="cuda")          # (what the next call's work memory holds)
    del junk
    for a, b in zip(first, both(q, k, v, dy, offsets=off, causal=True, cap=20.0)):
        assert torch.equal(a, b)


def test_a_part_of_the_gradients():
    g = gen(26)
    q, k, v, dy = normal(g, BF16, 300, 4, 256), normal(g, BF16, 300, 2, 256), normal(g, BF16, 300, 2, 256), normal(g, BF16, 300, 4, 256)
    y, lse, dq, dk, dv = both(q, k, v, dy, causal=True)
    for need, names in ((("q",), (dq, None, None)), (("k",), (None, dk, None)), (("v",), (None, None, dv)), (("k", "v"), (None, dk, dv)), ((), (None,) * 3)):
        got = B.alpa_attention_backward(dy, q, k, v, y, lse, causal=True, need=need)
        assert all((a is None) == (b is None) and (a is None or torch.equal(a, b)) for a, b in zip(got, names)), need
    room = torch.full((300, 10, 256), 3.0, dtype=BF16, device="cuda")
    out = room[:, :4], room[:, 4:6], room[:, 8:]
    assert B.alpa_attention_backward(dy, q, k, v, y, lse, causal=True, out=out)[1] is out[1]
    assert torch.equal(out[0], dq) and torch.equal(out[1], dk) and torch.equal(out[2], dv) and bool((room[:, 6:8] == 3.0).all())
    with pytest.raises(ValueError, match="out"):
        B.alpa_attention_backward(dy, q, k, v, y, lse, causal=True, out=(out[0], None, out[2]))


def leaves(*tensors):
    return [t.detach().clone().requires_grad_() for t in tensors]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_nodes_of_the_graph(dtype):
    """What torch's backward pass gives is what the calls themselves give: a block's first half with the heads as slices of one product's result."""
    g = gen(27)
    rows, n, kv, dim = 130, 4, 2, 32
    x, w, b = normal(g, dtype, rows, (n + 2 * kv) * dim), normal(g, dtype, (n + 2 * kv) * dim), normal(g, dtype, (n + 2 * kv) * dim)
    off, pos, f, dy = ints(0, 50, 130), torch.arange(rows, device="cuda"), B.alpa_rotary_frequencies(dim), normal(g, dtype, rows, n, dim)
    parts = lambda t: (t.view(rows, -1, dim)[:, :n], t.view(rows, -1, dim)[:, n:n + kv], t.view(rows, -1, dim)[:, n + kv:])
    # by hand
    h, mean, rstd = B.alpa_norm_forward(x, w, b, keep=True)
    q, k, v = parts(h)
    tq, tk = B.alpa_rotary_forward(q, pos, f), B.alpa_rotary_forward(k, pos, f)
    y, lse, *_ = both(tq, tk, v, dy, offsets=off, causal=True)
    dq, dk, dv = B.alpa_attention_backward(dy, tq, tk, v, y, lse, off, causal=True)
    dh = torch.cat([B.alpa_rotary_backward(dq, pos, f), B.alpa_rotary_backward(dk, pos, f), dv], 1).flatten(1)
    grads = B.alpa_norm_backward(dh, x, mean, rstd, w)
    # by torch, on this stream and on another one
    side = torch.cuda.Stream()
    for stream in (None, side):
        lx, lw, lb = leaves(x, w, b)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            hh = B.alpa_norm_forward(lx, lw, lb, stream=stream)
            qq, kk, vv = parts(hh)
            yy = B.alpa_attention_forward(B.alpa_rotary_forward(qq, pos, f, stream=stream), B.alpa_rotary_forward(kk, pos, f, stream=stream), vv, off, causal=True, stream=stream)
            yy.backward(dy)
        torch.cuda.synchronize()
        assert torch.equal(yy, y)
        for leaf, grad in zip((lx, lw, lb), grads):
            assert torch.equal(leaf.grad, grad)
    # a broadcast input's gradient is summed by torch over what it was broadcast to, and one number for all rows is handed over expanded
    lk, lv = leaves(tk[:, :1], v[:, :1])
    B.alpa_attention_forward(tq, lk.expand(-1, kv, -1), lv.expand(-1, kv, -1), off, causal=True).sum().backward()
    one = B.alpa_attention_forward(tq, tk[:, :1], v[:, :1], off, causal=True, keep_lse=True)
    _, dk1, dv1 = B.alpa_attention_backward(torch.ones_like(dy), tq, tk[:, :1], v[:, :1], *one, off, causal=True)
    for got, ref in ((lk.grad, dk1), (lv.grad, dv1)):
        assert float((got.to(D) - ref.to(D)).norm() / ref.to(D).norm()) <= 4 * {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -18}[dtype]


def test_what_is_not_recorded():
    x = torch.ones(4, 2, 8, device="cuda", requires_grad=True)
    y, lse = B.alpa_attention_forward(x, x, x, keep_lse=True)
    with pytest.raises(RuntimeError, match="lse has no gradient"):
        (y.sum() + lse.sum()).backward()
    with torch.no_grad():
        assert not B.alpa_attention_forward(x, x, x).requires_grad
    m = torch.ones(4, 8, device="cuda", requires_grad=True)
    h, mean, rstd = B.alpa_norm_forward(m, keep=True)
    with pytest.raises(RuntimeError, match="have no gradient"):
        (h.sum() + mean.sum()).backward()
    f, pos = B.alpa_rotary_frequencies(8), torch.arange(4, device="cuda")
    with pytest.raises(ValueError, match="recorded"):
        B.alpa_rotary_forward(x, pos, f, out=torch.empty_like(x))
    dx, = torch.autograd.grad(B.alpa_norm_forward(m).sum(), m, create_graph=True)
    with pytest.raises(RuntimeError):
        dx.sum().backward()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_calls_in_a_graph(dtype):
    """Two captured passes of their own work memory, replayed in turn with other work between: each replay gives what the calls give."""
    g = gen(28)
    shapes = ((1, 4096, 8, 2), (700, 700, 4, 2))
    state, graphs = [], []
    for rows, keys, n, kv in shapes:
        q, k, v, dy = normal(g, dtype, rows, n, 64), normal(g, dtype, keys, kv, 64), normal(g, dtype, keys, kv, 64), normal(g, dtype, rows, n, 64)
        pos, f, w = torch.arange(rows, device="cuda"), B.alpa_rotary_frequencies(64), normal(g, dtype, n * 64)

        def step(q=q, k=k, v=v, dy=dy, pos=pos, f=f, w=w):
            x = B.alpa_norm_forward(q.view(q.shape[0], -1), w, keep=True)
            t = B.alpa_rotary_forward(x[0].view_as(q), pos, f)
            r = both(t, k, v, dy, causal=True)
            return *r, *B.alpa_norm_backward(r[2].view(q.shape[0], -1), q.view(q.shape[0], -1), x[1], x[2], w)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        state.append((q, k, v, dy, step))
        graphs.append((graph, out))
    for turn in range(4):
        for (q, k, v, dy, step), (graph, out) in zip(state, graphs):
            for t in (q, k, v, dy):
                t.copy_(normal(g, dtype, *t.shape))
            graph.replay()
            torch.randn(1 << 20, device="cuda").sum().item()
        for (*_, step), (_, out) in zip(state, graphs):
            for a, b in zip(out, step()):
                assert torch.equal(a, b), turn


def test_two_streams_at_once():
    g = gen(29)
    sets = [[normal(g, BF16, 900, n, 64) for n in (8, 2, 2, 8)] for _ in range(2)]
    alone = [both(*s, causal=True) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for s, st in zip(sets, streams):
            y, lse = B.alpa_attention_forward(*s[:3], causal=True, keep_lse=True, stream=st)
            got.append((y, lse, *B.alpa_attention_backward(s[3], *s[:3], y, lse, causal=True, stream=st)))
        torch.cuda.synchronize()
        for a, b in zip(got, alone):
            assert all(torch.equal(x, z) for x, z in zip(a, b))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_norm_of_rows_that_do_not_vary(dtype):
    """A variance of zero leaves eps, large means leave no garbage in the variance, and infinities no numbers in their own rows alone."""
    x = torch.full((5, 700), 3.0, dtype=dtype, device="cuda")
    y, mean, rstd = B.alpa_norm_forward(x, eps=1e-5, keep=True)
    assert bool((y == 0).all()) and bool((mean == 3.0).all()) and bool(((rstd - 1e-5 ** -0.5).abs() <= 1e-4).all())
    x = (1000.0 + torch.arange(700, device="cuda") % 2 * 8.0).to(dtype).repeat(5, 1)
    ref = C.norm(x, None, None, 1e-5)
    C.within("y", B.alpa_norm_forward(x), ref["y"])
    x[2, 5] = math.inf
    y = B.alpa_norm_forward(x).float()
    assert not bool(torch.isfinite(y[2]).any()) and bool(torch.isfinite(y[[0, 1, 3, 4]]).all())


def test_many_rows():
    """Rows beyond what one launch has workgroups for, short ones; layer norm and rotary positions."""
    rows = (1 << 22) + 77
    x = torch.randn(rows, 8, device="cuda")
    y, mean, rstd = B.alpa_norm_forward(x, keep=True)
    at = torch.cat([torch.arange(100, device="cuda"), torch.arange(rows - 100, rows, device="cuda")])
    ref = C.norm(x[at], None, None, 1e-5)
    C.within("y", y[at], ref["y"])
    dx, _, db = B.alpa_norm_backward(torch.ones_like(x), x, mean, rstd)
    assert bool((db == rows).all())
    pos, f = torch.arange(rows, device="cuda"), B.alpa_rotary_frequencies(8)
    t = B.alpa_rotary_forward(x.view(rows, 1, 8), pos, f)
    C.within("t", t[at], C.rotary(x.view(rows, 1, 8)[at], pos[at], f, False, 1.0))


def test_rotary_of_wide_rows():
    """As many heads as allowed, as long as allowed, of which two elements are turned: more units than 32 bits count for 256 rows."""
    x = torch.empty(256, 4096, 4096, dtype=BF16, device="cuda").random_(-100, 100)
    pos, f = torch.arange(256, device="cuda"), B.alpa_rotary_frequencies(2)
    y = B.alpa_rotary_forward(x, pos, f)
    at = [0, 100, 255]
    C.within("y", y[at][:, ::1000], C.rotary(x[at][:, ::1000], pos[at], f, False, 1.0))
    assert torch.equal(y[..., 2:], x[..., 2:])


def test_positions_far_away():
    """Positions of 2^40 and negative ones: the angle is reduced in 64 bits."""
    g = gen(30)
    x, f = normal(g, F32, 6, 3, 64), B.alpa_rotary_frequencies(64)
    pos = torch.tensor([0, 1, -5, 1 << 31, (1 << 40) + 12345, -(1 << 40)], device="cuda")
    C.within("y", B.alpa_rotary_forward(x, pos, f), C.rotary(x, pos, f, False, 1.0))


def test_arguments_are_checked():
    q, k = torch.zeros(4, 6, 8, device="cuda", dtype=BF16), torch.zeros(4, 2, 8, device="cuda", dtype=BF16)
    for bad in (dict(k=k.float()), dict(k=k[:, :, :7]), dict(v=k[:3]), dict(k=k.cpu()), dict(offsets=torch.zeros(2, device="cuda")), dict(offsets=ints(0, 4), k_offsets=ints(0, 2, 4)),
                dict(k_offsets=ints(0, 2, 4)), dict(slopes=torch.zeros(5, device="cuda")), dict(prefix=ints(1, 2)), dict(q=q[0]), dict(q=q.transpose(1, 2))):
        with pytest.raises(ValueError):
            B.alpa_attention_forward(**{"q": q, "k": k, "v": k, **bad})
    for bad in (dict(cap=-1.0), dict(scale=math.inf), dict(q=q[:, :5])):
        with pytest.raises(Exception):
            B.alpa_attention_forward(**{"q": q, "k": k, "v": k, **bad})
    f, pos = B.alpa_rotary_frequencies(8), torch.arange(4, device="cuda")
    for bad in (dict(positions=pos.int()), dict(positions=pos[:3]), dict(frequencies=f.float()), dict(x=q[0])):
        with pytest.raises(ValueError):
            B.alpa_rotary_forward(**{"x": q, "positions": pos, "frequencies": f, **bad})
    with pytest.raises(Exception):
        B.alpa_rotary_forward(q, pos, torch.zeros(5, dtype=torch.float64, device="cuda"))
    m = torch.zeros(4, 8, device="cuda")
    for bad in (dict(weight=m[0, :7]), dict(bias=m[0].double()), dict(x=m.view(2, 2, 8))):
        with pytest.raises(ValueError):
            B.alpa_norm_forward(**{"x": m, **bad})
