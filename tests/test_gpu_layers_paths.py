"""Every compiled product on the device, at sizes listed with the path that they take (tests/layer_paths.py), against the definition
in 64 bits (bounds: tests/layer_cases.py)."""
import pytest
import torch

from paper_2201_12023_amd import layers as L
from tests import layer_cases as C
from tests import layer_paths as P

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def ends_of(rows, experts, g):
    """Uneven groups, one of them empty where there are several, rows of no expert on both sides."""
    cuts = torch.sort(torch.randint(rows // 50, rows - rows // 50 + 1, (experts + 1,), device="cuda", generator=g))[0].tolist()
    if experts > 2:
        cuts[1] = cuts[2]
    return cuts


def forward(dtype, act, rows, experts, n_in, n_out, g):
    many = () if experts < 0 else (experts,)
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, *many, n_out, n_in, scale=n_in ** -0.5)
    b, r = C.normal(g, dtype, *many, n_out), C.normal(g, dtype, rows, n_out)
    if experts < 0:
        y, z = L.alpa_linear_forward(x, w, b, r, act, keep_z=True)
        parts = [(slice(0, rows), w, b)]
    else:
        ends = ends_of(rows, experts, g)
        y, z = L.alpa_experts_forward(x, w, torch.tensor(ends, dtype=torch.int32, device="cuda"), b, r, act, keep_z=True)
        parts = [(slice(ends[e], ends[e + 1]), w[e], b[e]) for e in range(experts) if ends[e] < ends[e + 1]]
        for t in (y, z):
            assert not bool(t[:ends[0]].any()) and not bool(t[ends[-1]:].any())
    for p, we, be in parts:
        ry, ey, rz, ez = C.forward(x[p], we, be, r[p], act)
        C.within("y", y[p], ry, ey)
        C.within("z", z[p], rz, ez)


def backward(dtype, act, rows, experts, n_in, n_out, g):
    many = () if experts < 0 else (experts,)
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, *many, n_out, n_in, scale=n_in ** -0.5)
    dy, z = C.normal(g, dtype, rows, n_out), C.normal(g, dtype, rows, n_out)
    if experts < 0:
        got = L.alpa_linear_backward(dy, x, w, z if act else None, act)
        parts = [(slice(0, rows), w, got)]
    else:
        ends = ends_of(rows, experts, g)
        off = torch.tensor(ends, dtype=torch.int32, device="cuda")
        dx, dw, db = L.alpa_experts_backward(dy, x, w, off, z if act else None, act)
        assert not bool(dx[:ends[0]].any()) and not bool(dx[ends[-1]:].any())
        parts = []
        for e in range(experts):
            if ends[e] < ends[e + 1]:
                parts.append((slice(ends[e], ends[e + 1]), w[e], (dx[ends[e]:ends[e + 1]], dw[e], db[e])))
            else:
                assert not bool(dw[e].any()) and not bool(db[e].any())
    for p, we, results in parts:
        ref = C.backward(dy[p], z[p], x[p], we, act)
        for name, t in zip(("dx", "dw", "dbias"), results):
            C.within(name, t, *ref[name])


def loss(dtype, act, rows, experts, n_in, words, g, gradient=False):
    x, w = C.normal(g, dtype, rows, n_in), C.normal(g, dtype, words, n_in, scale=n_in ** -0.5)
    t = torch.randint(0, words, (rows,), device="cuda", generator=g)
    if rows > 1:
        t[torch.rand(rows, device="cuda", generator=g) < 0.1] = -100
    dloss = torch.rand(rows, device="cuda", generator=g) + 0.5
    ref = C.vocab(x, w, t, dloss if gradient else None)
    value, lse = L.alpa_vocab_loss_forward(x, w, t)
    C.within("loss", value, *ref["loss"])
    C.within("lse", lse, *ref["lse"])
    if gradient:
        dx, dw = L.alpa_vocab_loss_backward(dloss, x, w, t, lse)
        C.within("dx", dx, *ref["dx"])
        C.within("dw", dw, *ref["dw"])


def gradient(*args):
    loss(*args, gradient=True)


@pytest.mark.parametrize("dtype", [BF16, F16, F32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("path, small, wide", P.PATHS, ids=["-".join(map(str, p[0])) for p in P.PATHS])
def test_path(path, small, wide, dtype):
    name, *sizes = wide if dtype == F32 else small
    {"forward": forward, "backward": backward, "loss": loss, "gradient": gradient}[name](dtype, *sizes, C.gen(61))
