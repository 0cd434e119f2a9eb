"""Attention where numbers end: scores that are no number under a cap, caps far above the scores, and weights below what float16 holds."""
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


# (rows, keys, heads, kv heads, dim, offsets, key offsets): few rows and keys in tiles of 128; tiles of many rows and keys in tiles of 256; heads above 128
SHAPES = [(130, 130, 4, 2, 64, (0, 40, 80, 120), (0, 40, 80, 120)), (1815, 2000, 20, 20, 64, (7, 607, 1807), (2, 777, 1990)), (90, 100, 4, 2, 200, (0, 90), (0, 100))]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:5])))
@pytest.mark.parametrize("cap, slopes", [(30.0, False), (30.0, True), (1e5, False), (0.0, True)])
def test_a_score_that_is_no_number_stays_none(dtype, shape, cap, slopes):
    """A NaN in a row of q, or in a key, is one in y, lse and dq of the rows that see it, and in the gradients of what they see; other sequences and kv heads keep their bits."""
    rows, k_rows, heads, kv, dim, off, k_off = shape
    g, group = gen(41), heads // kv
    q, k, v, dy = normal(g, dtype, rows, heads, dim), normal(g, dtype, k_rows, kv, dim), normal(g, dtype, k_rows, kv, dim), normal(g, dtype, rows, heads, dim)
    how = dict(offsets=ints(*off), k_offsets=ints(*k_off), causal=True, cap=cap, slopes=torch.linspace(0.01, 0.5, heads, device="cuda") if slopes else None)
    clean = both(q, k, v, dy, **how)
    s = len(off) - 2                                       # the last sequence
    a, b, c, e = off[s], off[s + 1], k_off[s], k_off[s + 1]
    nan = lambda t: bool(torch.isnan(t).all())

    def others(got):
        for t, ref in zip(got, clean):
            kept = torch.ones_like(ref, dtype=torch.bool)
            first, last = (a, b) if ref.shape[0] == rows and ref.shape[1] == heads else (c, e)
            kept[first:last, :group if ref.shape[1] == heads else 1] = False
            assert torch.equal(t[kept], ref[kept])
    # a row: it sees the keys up to its own place
    i = b - 10
    last = c + (i - a) + (e - c) - (b - a)
    was = q[i, 0].clone()
    q[i, 0, dim // 2] = math.nan
    y, lse, dq, dk, dv = got = both(q, k, v, dy, **how)
    q[i, 0] = was
    assert nan(y[i, 0]) and nan(lse[i, 0]) and nan(dq[i, 0]) and nan(dk[c:last + 1, 0]) and nan(dv[c:last + 1, 0])
    # the rows of this head and sequence beside it are what they were but for roundings (when sums are brought to a new reference is up to all rows of a tile)
    rest = torch.arange(a, b, device="cuda") != i
    near = lambda x, ref: float((x.float() - ref.float()).abs().max()) <= 2.0 ** -5
    assert near(y[a:b, 0][rest], clean[0][a:b, 0][rest]) and near(lse[a:b, 0][rest], clean[1][a:b, 0][rest])
    others(got)
    # a key
    j = e - 20
    k[j, 0, 1] = math.nan
    y, lse, dq, dk, dv = got = both(q, k, v, dy, **how)
    first = b - 20                                         # (the last row meets the last key)
    assert nan(y[first:b, :group]) and nan(lse[first:b, :group]) and nan(dq[first:b, :group]) and nan(dk[j, 0])
    assert near(y[a:first, :group], clean[0][a:first, :group]) and near(lse[a:first, :group], clean[1][a:first, :group])
    others(got)
    # all keys: no score is a number
    k[c:e, 0] = math.nan
    y, lse, dq, dk, dv = got = both(q, k, v, dy, **how)
    assert nan(y[a:b, :group]) and nan(lse[a:b, :group]) and nan(dq[a:b, :group]) and nan(dk[c:e, 0])
    others(got)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, heads, kv", [(90, 4, 2), (2000, 20, 20)])
@pytest.mark.parametrize("cap", [1e5, 1e8, 3e38])
def test_caps_far_above_the_scores(dtype, rows, heads, kv, cap):
    """Scores of up to 8 under a cap of 1e5 and more are what they are without one to 8^3 / (3 cap^2) = 2e-8, which the bounds without a cap leave room for (4 * 2^-23 a score).
    The slope of the cap, 1 to 2e-8, is known to 6 units of 2^-23, a hundredth of the roundings to 16 bits that the bounds of the gradients count, and a sixtieth of the products'
    of 64 terms in 32 bits."""
    g = gen(42)
    q, k, v, dy = normal(g, dtype, rows, heads, 64), normal(g, dtype, rows, kv, 64), normal(g, dtype, rows, kv, 64), normal(g, dtype, rows, heads, 64)
    assert float(torch.matmul(q[:, :1].transpose(0, 1).float(), k[:, 0].float().t()).abs().max()) / 8.0 < 8.0
    ref = C.attention(q, k, v, dy, causal=True)
    for name, got in zip(("y", "lse", "dq", "dk", "dv"), both(q, k, v, dy, causal=True, cap=cap)):
        value, bound = ref[name]
        C.within(name, got, (value, bound * (1.02 if name in ("dq", "dk") else 1.0)))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("cap", [1e-30, 1e-3, 0.5, 255.0, 257.0, 1000.0])
@pytest.mark.parametrize("reach", [0.2, 3.0])
def test_caps_of_all_sizes(dtype, cap, reach):
    """Scores from far below the cap to several times it."""
    g = gen(43)
    q, k, v, dy = (normal(g, dtype, 70, n, 64) for n in (4, 2, 2, 4))
    how = dict(causal=True, cap=cap, scale=cap * reach / 8.0)
    ref = C.attention(q, k, v, dy, **how)
    for name, got in zip(("y", "lse", "dq", "dk", "dv"), both(q, k, v, dy, **how)):
        C.within(name, got, ref[name])


def test_a_cap_whose_inverse_overflows():
    """2 scale / cap beyond 32 bits: a score of zero is zero, the others are at the cap, too small to count: all keys weigh the same."""
    for dtype in TYPES:
        q, k = torch.zeros(3, 1, 64, device="cuda", dtype=dtype), normal(gen(44), dtype, 50, 1, 64)
        q[1, 0, 0] = 1.0
        v = normal(gen(45), dtype, 50, 1, 64)
        y, lse = B.alpa_attention_forward(q, k, v, cap=1e-39, scale=1.0, keep_lse=True)
        mean = v[:, 0].to(D).mean(0)
        # 50 values in 32 bits, one rounding
        assert bool(((y[:, 0].to(D) - mean).abs() <= 60 * 2.0 ** -23 * v.to(D).abs().amax() + {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 0.0}[dtype] * mean.abs()).all())
        assert bool(((lse - math.log(50.0)).abs() <= 1e-5).all())


@pytest.mark.parametrize("keys, dim", [(100003, 64), ((1 << 25) + 3, 8)])
def test_gradients_of_weights_that_float16_does_not_hold(keys, dim):
    """Rows of zeros weigh all keys alike, by 1 / keys, which float16 has with 8 bits (1e-5) or not at all (2^-25).  dv = sum(dy) / keys for each key, of an ordinary size.
    A weight's exponent, up to 26, is off by 4 units of 2^-23 of it: 1.3e-5; the weight is rounded once and dv once, 2^-11 each; 32 terms are summed in 32 bits."""
    g, rows = gen(46), 32
    k, v = normal(g, F16, keys, 1, dim), normal(g, F16, keys, 1, dim)
    q = torch.zeros(rows, 1, dim, device="cuda", dtype=F16)
    dy = ((1.0 + torch.rand(rows, 1, dim, device="cuda", generator=g)) * (keys / 4096.0)).clamp(max=30000.0).to(F16)
    y, lse = B.alpa_attention_forward(q, k, v, keep_lse=True)
    assert bool(((lse - math.log(keys)).abs() <= 1e-4).all())
    dv = B.alpa_attention_backward(dy, q, k, v, y, lse, need=("v",))[2]
    ref = dy[:, 0].to(D).sum(0) / keys
    assert float(ref.min()) > 2.0 ** -9
    off = ((dv[:, 0].to(D) - ref).abs() / ref).amax()
    assert float(off) <= 2 * 2.0 ** -11 + 1e-4, float(off)


@pytest.mark.parametrize("rows", [3, 76900])
def test_many_small_weights_beside_a_large_one_in_float16(rows):
    """One key has a score of 0, the others 17.5 less: each weighs 2^-25.2, 131071 of them 0.0033 together, which is y where the first key's value is 0 and theirs 1.
    The weights are rounded once (2^-11), y once; their exponents, up to 26, are off by 4 units of 2^-23 of them; and what y is divided by, a sum in 32 bits, may lose the
    small weights beside the large one, 0.0033 of it.  With few rows the weights are relative to each wave's own largest, with many rows to the first key's."""
    keys = 1 << 17
    q, k = torch.zeros(rows, 1, 8, device="cuda", dtype=F16), torch.zeros(keys, 1, 8, device="cuda", dtype=F16)
    q[..., 0] = 1.0
    k[1:, 0, 0] = -17.5
    v = torch.ones(keys, 1, 8, device="cuda", dtype=F16)
    v[0] = 0.0
    y = B.alpa_attention_forward(q, k, v, scale=1.0)
    total = (keys - 1) * math.exp(-17.5)
    ref = total / (1.0 + total)
    assert float((y.to(D) - ref).abs().max()) <= ref * (2 * 2.0 ** -11 + total + 2e-5)
