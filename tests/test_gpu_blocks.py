"""Attention, rotary positions and layer norm against their definitions in 64 bits, within bounds derived from the arithmetic (tests/block_cases.py)."""
import itertools

import pytest
import torch

from paper_2201_12023_amd import blocks as B
from tests import block_cases as C
from tests.layer_cases import gen, normal

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [BF16, F16, F32]


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def check_attention(g, dtype, rows, k_rows, heads, kv_heads, dim, train=True, size=1.0, **how):
    q, k, v = normal(g, dtype, rows, heads, dim, scale=size), normal(g, dtype, k_rows, kv_heads, dim, scale=size), normal(g, dtype, k_rows, kv_heads, dim)
    dy = normal(g, dtype, rows, heads, dim) if train else None
    ref = C.attention(q, k, v, dy, **how)
    y, lse = B.alpa_attention_forward(q, k, v, keep_lse=True, **how)
    C.within("y", y, ref["y"])
    C.within("lse", lse, ref["lse"])
    if train:
        for name, got in zip(("dq", "dk", "dv"), B.alpa_attention_backward(dy, q, k, v, y, lse, **how)):
            C.within(name, got, ref[name])
    return q, k, v, dy, y, lse


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, keys", [(1, 1), (1, 2), (1, 31), (3, 33), (31, 64), (32, 65), (64, 64), (65, 127), (129, 129), (200, 333), (300, 300)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(dtype, rows, keys, causal):
    check_attention(gen(rows * 1000 + keys), dtype, rows, keys, 4, 2, 64, causal=causal)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim", [1, 2, 7, 8, 16, 33, 64, 65, 75, 80, 96, 97, 128, 129, 160, 192, 250, 256])
def test_head_sizes(dtype, dim):
    check_attention(gen(dim), dtype, 150, 150, 2, 2, dim, causal=True)


@pytest.mark.parametrize("heads, kv_heads", [(1, 1), (3, 3), (3, 1), (8, 1), (8, 2), (10, 2), (40, 1), (35, 5)])
@pytest.mark.parametrize("rows, keys", [(1, 70), (5, 5), (90, 130)])
def test_head_groups(heads, kv_heads, rows, keys):
    check_attention(gen(heads), BF16, rows, keys, heads, kv_heads, 64, causal=True)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("causal, prefix", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("cap, slopes", [(0.0, False), (5.0, False), (0.0, True), (20.0, True)])
def test_masks_and_scores(dtype, causal, prefix, cap, slopes):
    """Packed sequences, empty ones among them, rows and keys of none around them, sequences with more keys than rows and with fewer, which leave rows without keys."""
    g = gen(3)
    off, k_off = ints(2, 2, 40, 41, 90, 230), ints(3, 9, 70, 70, 190, 260)
    check_attention(g, dtype, 240, 270, 6, 2, 64, offsets=off, k_offsets=k_off, causal=causal, prefix=ints(5, 0, 3, 200, 17) if prefix else None, cap=cap,
                    slopes=torch.tensor([0.5, 0.25, 0.0, 0.1, 1.0, -0.01], device="cuda") if slopes else None, size=2.0)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_scales(dtype, scale):
    check_attention(gen(4), dtype, 70, 90, 2, 2, 64, scale=scale, causal=True)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("new, group", [(1, 1), (1, 8), (2, 5), (4, 16), (7, 12)])
def test_new_tokens_over_a_cache(dtype, new, group):
    """Caches of unequal length with room behind them that holds no numbers, one of them empty, in places out of order."""
    g = gen(new)
    lens, most, kv, dim = [500, new, 0, 127, 128, 300], 512, 2, 128
    order = [3, 0, 5, 1, 2, 4]
    seqs = len(lens)
    k, v = (normal(g, dtype, seqs * most, kv, dim) for _ in range(2))
    pairs = ints(*[[o * most, o * most + n] for o, n in zip(order, lens)])
    for o, n in zip(order, lens):
        k[o * most + n:(o + 1) * most] = float("nan")
        v[o * most + n:(o + 1) * most] = float("nan")
    q = normal(g, dtype, seqs * new, kv * group, dim)
    off = torch.arange(seqs + 1, device="cuda", dtype=torch.int32) * new
    ref = C.attention(q, k, v, None, offsets=off, k_offsets=pairs, causal=True)
    y, lse = B.alpa_attention_forward(q, k, v, off, pairs, causal=True, keep_lse=True)
    C.within("y", y, ref["y"])
    C.within("lse", lse, ref["lse"])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, keys, heads, kv", [(1, 40000, 4, 1), (300, 9000, 2, 1), (17, 2000, 64, 1)])
def test_few_rows_with_many_keys(dtype, rows, keys, heads, kv):
    """Keys in parts that are joined, for one row and for tiles of rows."""
    check_attention(gen(9), dtype, rows, keys, heads, kv, 64, train=False, causal=True)


@pytest.mark.parametrize("keys", [1, 70])
def test_very_many_sequences(keys):
    """One row of each of 700 sequences, some without keys, rows of none on both sides."""
    g, seqs = gen(11), 700
    lens = torch.randint(0, keys + 1, (seqs,), device="cuda", generator=g, dtype=torch.int32)
    ends = torch.cumsum(lens, 0).to(torch.int32)
    k_off = torch.cat([torch.zeros_like(ends[:1]), ends])
    off = torch.arange(seqs + 1, device="cuda", dtype=torch.int32) + 2
    check_attention(g, BF16, seqs + 7, int(ends[-1]) + 3, 4, 2, 64, offsets=off, k_offsets=k_off, causal=True)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_tiles_of_many_rows(dtype, causal):
    """Enough rows for the kernels that share tiles of keys among rows, forward and backward."""
    off = ints(1, 1300, 1300, 2000, 2950)
    check_attention(gen(12), dtype, 2960, 2960, 24, 12, 64, offsets=off, causal=causal, cap=8.0 if causal else 0.0)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("dim, extra", [(64, True), (80, False), (128, False), (128, True)])
def test_tiles_of_256_keys(dtype, dim, extra):
    """Long sequences of many kv heads: keys in tiles of 256, of which some end inside, behind rows and keys of no sequence."""
    off, k_off = ints(7, 607, 1807), ints(2, 777, 1990)
    slopes = torch.linspace(0.01, 0.5, 20, device="cuda") if extra else None
    check_attention(gen(13), dtype, 1815, 2000, 20, 20, dim, offsets=off, k_offsets=k_off, causal=True, prefix=ints(300, 0), cap=10.0 if extra else 0.0, slopes=slopes)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_many_rows_with_few_keys(dtype):
    """Gradients of keys whose rows go in parts that are added."""
    check_attention(gen(10), dtype, 700, 60, 16, 1, 96, causal=False)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows, heads, dim, rot", [(1, 1, 2, 2), (1, 40, 128, 128), (5, 3, 80, 20), (70, 7, 75, 30), (33, 2, 64, 64), (3, 2, 256, 128), (4, 1, 4096, 4096)])
def test_rotary(dtype, interleaved, rows, heads, dim, rot):
    g = gen(rot)
    x = normal(g, dtype, rows, heads + 2, dim)[:, 1:heads + 1]
    pos = torch.randint(0, 1 << 20, (rows,), device="cuda", generator=g)
    f = B.alpa_rotary_frequencies(rot)
    for scale in (1.0, 1.3):
        C.within("y", B.alpa_rotary_forward(x, pos, f, interleaved, scale), C.rotary(x, pos, f, interleaved, scale))
        C.within("dx", B.alpa_rotary_backward(x, pos, f, interleaved, scale), C.rotary(x, pos, f, interleaved, scale, back=True))
    at = x.clone(memory_format=torch.contiguous_format)
    assert B.alpa_rotary_forward(at, pos, f, interleaved, out=at) is at
    assert torch.equal(at, B.alpa_rotary_forward(x, pos, f, interleaved))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, n", [(1, 1), (2, 8), (5, 100), (70, 512), (3, 1001), (40, 1024), (9, 2048), (30, 4096), (17, 5000), (6, 8192), (5, 16384),
                                     (3, 16392), (2, 40000)])
@pytest.mark.parametrize("weight, bias", [(False, False), (True, True)])
def test_norm(dtype, rows, n, weight, bias):
    g = gen(n)
    x = (torch.randn(rows, n, device="cuda", generator=g) * 2 + 1).to(dtype)
    w, b = normal(g, dtype, n) if weight else None, normal(g, dtype, n) if bias else None
    dy = normal(g, dtype, rows, n)
    ref = C.norm(x, w, b, 1e-5, dy)
    y, mean, rstd = B.alpa_norm_forward(x, w, b, keep=True)
    got = {"y": y, "mean": mean, "rstd": rstd, **dict(zip(("dx", "dweight", "dbias"), B.alpa_norm_backward(dy, x, mean, rstd, w)))}
    for name, value in got.items():
        C.within(name, value, ref[name])


@pytest.mark.parametrize("dtype,n", [(BF16, 72), (BF16, 1000), (F16, 1024), (BF16, 2049), (BF16, 4096), (F16, 4095), (BF16, 8192), (BF16, 10001), (F32, 65), (F32, 1001), (F32, 2048)])
@pytest.mark.parametrize("rows", [511, 513, 1025, 2047, 2055])
def test_gradients_of_norm_rows_that_share_a_workgroup(dtype, n, rows):
    """A workgroup takes some rows at once, the last of them not in all of its threads; what one of dx, dweight and dbias is does not depend on the others."""
    g = gen(rows * 7 + n)
    x, dy, w = normal(g, dtype, rows, n), normal(g, dtype, rows, n), normal(g, dtype, n)
    ref = C.norm(x, w, None, 1e-5, dy)
    _, mean, rstd = B.alpa_norm_forward(x, w, keep=True)
    got = B.alpa_norm_backward(dy, x, mean, rstd, w)
    for name, t in zip(("dx", "dweight", "dbias"), got):
        C.within(name, t, ref[name])
    for i, name in enumerate(("x", "weight", "bias")):
        assert torch.equal(B.alpa_norm_backward(dy, x, mean, rstd, w, need=(name,))[i], got[i])
