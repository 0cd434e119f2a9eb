"""CPU-side checks of the C ABI of attention, rotary positions and layer norm: exported symbols, refusals before a device is touched, and what is computed on the
host."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2201_12023_amd import blocks as B
from paper_2201_12023_amd import layers as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20          # an address that is never followed: every call here is refused, or has nothing to do
NONE = B.alpa_heads_t(None, 0, 0)


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "alpa_blocks.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(alpa_[a-z_]+)\s*\(", text))
    assert names == set(B.SYMBOLS)
    lib = B.load()
    for n in names:
        assert hasattr(lib, n), n


def H(p, row, head):
    return B.alpa_heads_t(p, row, head)


Q, K = H(P, 4 * 64, 64), H(P, 2 * 64, 64)


def how(dtype=2, seqs=1, heads=4, kv_heads=2, dim=64, causal=1, k_step=1, scale=0.125, cap=0.0, rows=5, k_rows=7, offsets=P, k_offsets=P, prefix=None, slopes=None):
    return B.alpa_attention_t(dtype, seqs, heads, kv_heads, dim, causal, k_step, scale, cap, rows, k_rows, offsets, k_offsets, prefix, slopes)


def forward(q=Q, k=K, v=K, y=Q, lse=None, work=None, n=0, **over):
    return B.load().alpa_attention_forward(how(**over), q, k, v, y, lse, work, n, None)


def backward(dy=Q, q=Q, k=K, v=K, y=Q, lse=P, dq=Q, dk=K, dv=K, work=P, n=1 << 30, **over):
    return B.load().alpa_attention_backward(how(**over), dy, q, k, v, y, lse, dq, dk, dv, work, n, None)


BAD = [dict(dtype=3), dict(dtype=-1), dict(seqs=0), dict(seqs=B.ATTENTION_MAX_SEQS + 1), dict(heads=0), dict(heads=5), dict(heads=B.MAX_HEADS * 2), dict(kv_heads=0),
       dict(dim=0), dict(dim=257), dict(k_step=0), dict(k_step=3), dict(scale=math.inf), dict(scale=math.nan), dict(cap=-1.0), dict(cap=math.nan), dict(rows=-1),
       dict(rows=1 << 29), dict(k_rows=-1), dict(rows=(1 << 28) + 1, heads=4), dict(rows=1 << 28, heads=8), dict(offsets=P + 2), dict(k_offsets=P + 1), dict(prefix=P + 1), dict(slopes=P + 3),
       dict(offsets=None, seqs=2), dict(k_offsets=None, seqs=2), dict(q=NONE), dict(k=NONE), dict(v=NONE), dict(y=NONE), dict(q=H(P + 1, 256, 64)),
       dict(q=H(P, -256, 64)), dict(k=H(P, 128, (1 << 40) + 1)), dict(lse=P + 2)]


@pytest.mark.parametrize("bad", BAD, ids=lambda b: "-".join(b))
def test_attention_refuses(bad):
    assert forward(**bad) == -1
    assert backward(**bad) == -1
    sizes = {k: v for k, v in bad.items() if k not in ("q", "k", "v", "y", "lse")}
    if sizes:
        assert B.load().alpa_attention_forward_work(how(**sizes), Q, K, K) == 0
        assert B.load().alpa_attention_backward_work(how(**sizes), Q, Q, K, K, Q) == 0


@pytest.mark.parametrize("y", [H(P, 4 * 64, 63), H(P, 4 * 64 - 1, 64), H(P, 0, 64), H(P, 63, 5 * 64)])
def test_results_that_overlap_are_refused(y):
    assert forward(y=y) == -1 and backward(dq=y) == -1
    assert b"overlap" in B.load().alpa_dp_last_error()


def test_attention_needs_its_memory():
    assert forward(rows=0, q=NONE, y=NONE) == 0                              # nothing to do
    need = B.load().alpa_attention_forward_work(how(k_rows=5000), Q, K, K)        # few rows with many keys: in parts
    assert need > 0
    assert forward(k_rows=5000) == -1 and forward(k_rows=5000, work=P, n=need - 1) == -1 and forward(k_rows=5000, work=P + 64, n=need) == -1
    assert B.load().alpa_attention_forward_work(how(), Q, K, K) == 0
    # copies of what is not aligned to 16 bytes
    odd = B.load().alpa_attention_forward_work(how(dim=63), Q, K, K)
    assert odd == 5 * 4 * 64 * 2 + 2 * (7 * 2 * 64 * 2)
    assert B.load().alpa_attention_forward_work(how(), H(P + 2, 256, 64), K, K) == 5 * 4 * 64 * 2
    assert backward(n=16) == -1 and backward(work=None) == -1
    assert backward(lse=None) == -1 and backward(dy=NONE) == -1 and backward(k_step=2) == -1
    assert B.load().alpa_attention_backward_work(how(k_step=2), Q, Q, K, K, Q) == 0


def rotary(dtype=2, rows=3, heads=2, dim=8, rot=8, inter=0, scale=1.0, pos=P, f=P, x=H(P, 16, 8), y=H(2 * P, 16, 8)):
    return [fn(dtype, rows, heads, dim, rot, inter, scale, pos, f, x, y, None) for fn in (B.load().alpa_rotary_forward, B.load().alpa_rotary_backward)]


@pytest.mark.parametrize("bad", [dict(dtype=7), dict(rows=-1), dict(rows=(1 << 28) + 1), dict(heads=0), dict(heads=B.MAX_HEADS + 1), dict(dim=1), dict(dim=B.MAX_DIM + 1),
                                 dict(rot=0), dict(rot=7), dict(rot=10), dict(scale=math.inf), dict(pos=None), dict(f=None), dict(pos=P + 4), dict(f=P + 4), dict(x=NONE), dict(y=NONE),
                                 dict(x=H(P + 1, 16, 8)), dict(y=H(2 * P, 16, 7)), dict(y=H(2 * P, 15, 8)), dict(y=H(P, 32, 8))], ids=lambda b: "-".join(b))
def test_rotary_refuses(bad):
    assert rotary(**bad) == [-1, -1]


def test_rotary_of_nothing():
    assert rotary(rows=0, x=NONE, y=NONE, pos=None, f=None) == [0, 0]


def test_frequencies():
    f = B.alpa_rotary_frequencies(64, base=500000.0, device="cpu")
    ref = 500000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    assert torch.allclose(f, ref, rtol=1e-13, atol=0.0)
    assert torch.allclose(B.alpa_rotary_frequencies(64, base=500000.0, factor=8.0, device="cpu"), ref / 8, rtol=1e-13, atol=0.0)
    f = B.alpa_rotary_frequencies(64, base=500000.0, factor=8.0, context=8192, low=1.0, high=4.0, device="cpu")
    turns = 8192 * ref / (2 * math.pi)
    kept = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
    assert torch.allclose(f, ref * kept + ref / 8 * (1 - kept), rtol=1e-13, atol=0.0)
    assert bool((f[turns >= 4] == ref[turns >= 4]).all()) and bool((kept > 0).any()) and bool(((kept > 0) & (kept < 1)).any())


@pytest.mark.parametrize("bad", [dict(rot=0), dict(rot=3), dict(rot=-2), dict(rot=B.MAX_DIM + 2), dict(base=0.0), dict(base=math.inf), dict(factor=0.0), dict(factor=-1.0),
                                 dict(context=-1.0), dict(context=math.nan), dict(context=8.0, low=4.0, high=4.0)], ids=lambda b: "-".join(b))
def test_frequencies_refuse(bad):
    with pytest.raises(Exception):
        B.alpa_rotary_frequencies(**{"rot": 8, "device": "cpu", **bad})


M = L.alpa_mat_t


def norm(dtype=2, rows=3, n=8, eps=1e-5, x=M(P, 8), w=None, b=None, y=M(P, 8), mean=None, rstd=None):
    return B.load().alpa_norm_forward(dtype, rows, n, eps, x, w, b, y, mean, rstd, None)


def norm_backward(dtype=2, rows=3, n=8, dy=M(P, 8), x=M(P, 8), mean=P, rstd=P, w=None, dx=M(P, 8), dw=P, db=P, work=P, size=1 << 20):
    return B.load().alpa_norm_backward(dtype, rows, n, dy, x, mean, rstd, w, dx, dw, db, work, size, None)


def test_norm_refuses():
    for bad in (dict(dtype=3), dict(rows=-1), dict(rows=L.MAX_ROWS + 1), dict(n=0), dict(n=L.MAX_WIDTH + 1), dict(x=M(None, 8)), dict(x=M(P, 7)), dict(x=M(P + 1, 8)), dict(w=P + 1)):
        assert norm(**bad) == -1 and norm_backward(**bad) == -1, bad
    for bad in (dict(eps=-1.0), dict(eps=math.nan), dict(y=M(None, 8)), dict(b=P + 1), dict(mean=P), dict(rstd=P), dict(mean=P + 2, rstd=P)):
        assert norm(**bad) == -1, bad
    for bad in (dict(dy=M(None, 8)), dict(mean=None), dict(rstd=None), dict(dx=M(P, 7)), dict(dw=P + 1), dict(db=P + 1), dict(work=None), dict(size=8), dict(work=P + 8)):
        assert norm_backward(**bad) == -1, bad
    assert norm(rows=0, x=M(None, 0), y=M(None, 0)) == 0
    assert norm_backward(rows=0, dw=None, db=None, x=M(None, 0), dy=M(None, 0), dx=M(None, 0)) == 0
    assert B.load().alpa_norm_backward_work(3, 1, 8) == 0 and B.load().alpa_norm_backward_work(2, 1, 0) == 0


def test_python_refuses_before_the_library():
    x = torch.zeros(4, 2, 8)
    with pytest.raises(ValueError, match="GPU"):
        B.alpa_attention_forward(x, x, x)
    with pytest.raises(ValueError, match="GPU"):
        B.alpa_rotary_forward(x, torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.float64))
    with pytest.raises(ValueError, match="GPU"):
        B.alpa_norm_forward(torch.zeros(4, 8))
    with pytest.raises(ValueError, match="type"):
        B.alpa_norm_forward(torch.zeros(4, 8, dtype=torch.float64))
    with pytest.raises(ValueError, match="need"):
        B.alpa_attention_backward(x, x, x, x, x, x, need=("w",))
    with pytest.raises(ValueError, match="packed"):
        B.alpa_attention_backward(x, x, x, x, x, x, k_offsets=torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="slopes"):
        B.alpa_attention_forward(x, x, x, slopes=torch.zeros(2, requires_grad=True))
    with pytest.raises(ValueError, match="packed"):
        B.alpa_attention_forward(x.clone().requires_grad_(), x, x, k_offsets=torch.zeros(1, 2, dtype=torch.int32))
