"""Every compiled kernel of attention on the device, at shapes listed with the path that they take (tests/block_paths.py), against the definition in 64 bits (bounds:
tests/block_cases.py)."""
import pytest
import torch

from paper_2201_12023_amd import blocks as B
from tests import block_cases as C
from tests import block_paths as P
from tests.layer_cases import D, gen, normal

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def ends(lens, slack):
    """Offsets, with rows of no sequence on both sides."""
    first = slack // 2
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


# (caps of all sizes are one kernel in 32 bits)
@pytest.mark.parametrize("dtype, score", [(t, s) for t in (BF16, F16, F32) for s in P.CAPS if t != F32 or s != "far"], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("blocks", list(P.DIMS))
@pytest.mark.parametrize("name", list(P.SHAPES))
def test_path(name, dtype, blocks, score):
    s, dim, g = P.SHAPES[name], P.DIMS[blocks], gen(71)
    q, k, v, dy = normal(g, dtype, s.rows, s.heads, dim), normal(g, dtype, s.k_rows, s.kv_heads, dim), normal(g, dtype, s.k_rows, s.kv_heads, dim), normal(g, dtype, s.rows, s.heads, dim)
    how = dict(offsets=ends(s.lens, s.rows - sum(s.lens)), k_offsets=ends(s.k_lens, s.k_rows - sum(s.k_lens)), scale=0.125, cap=P.CAPS[score], causal=s.causal,
               slopes=torch.linspace(-0.01, 0.3, s.heads, device="cuda") if score != "plain" else None,
               prefix=None if s.prefix is None else torch.tensor(s.prefix, dtype=torch.int32, device="cuda"))
    ref = C.attention(q, k, v, dy, **how)
    y, lse = B.alpa_attention_forward(q, k, v, keep_lse=True, **how)
    for name, got in zip(("y", "lse", "dq", "dk", "dv"), (y, lse, *B.alpa_attention_backward(dy, q, k, v, y, lse, **how))):
        C.within(name, got, ref[name])


def lse_bound(Q, K, a):
    """of two scores of 8 products each, in 32 bits"""
    return 2.0 ** -23 * (12 * 0.3 * (Q * K).abs().sum(-1).amax(1) + 4 * a.abs().amax(1) + 20)


def test_more_workgroups_than_a_launch_has():
    """4.2 million tiles of one row each (and of two keys): a sequence of one row and two keys for each of 1030 times 4096 heads."""
    g, seqs, n = gen(72), 1030, 4096
    q, k, v, dy = (normal(g, BF16, m, n, 8) for m in (seqs, 2 * seqs, 2 * seqs, seqs))
    off = torch.arange(seqs + 1, device="cuda", dtype=torch.int32)
    y, lse = B.alpa_attention_forward(q, k, v, off, 2 * off, scale=0.3, keep_lse=True)
    dq, dk, dv = B.alpa_attention_backward(dy, q, k, v, y, lse, off, 2 * off, scale=0.3)
    pairs = lambda t: t.view(seqs, 2, n, 8)
    Q, K, V, E = q.to(D)[:, None], pairs(k).to(D), pairs(v).to(D), dy.to(D)[:, None]
    a = 0.3 * (Q * K).sum(-1)
    p = torch.softmax(a, 1)[..., None]
    Y = (p * V).sum(1, keepdim=True)
    d = 0.3 * p * ((E * V).sum(-1, keepdim=True) - (E * Y).sum(-1, keepdim=True))
    # Two weights rounded to bfloat16 (u = 2^-8) and divided by their sum leave y off by p1 p2 2 u |v1 - v2| <= u max|v|, its own rounding by u |y|; dy . y of it by 2 u sum |dy| max|v|;
    # dR is rounded once, its products' sum once, each at most u of `size`
    size = (E * V).abs().sum(-1, keepdim=True) + (E.abs() * V.abs().amax(1, keepdim=True)).sum(-1, keepdim=True)
    for got, ref, most in ((y, Y[:, 0], V.abs().amax(1)), (dv, p * E, E.abs().expand_as(p * E)), (dk, d * Q, 0.3 * size * Q.abs()), (dq, (d * K).sum(1), 0.3 * (size * K.abs()).sum(1))):
        got = pairs(got) if got.shape[0] == 2 * seqs else got
        assert bool(((got.to(D) - ref).abs() <= 4 * 2.0 ** -8 * most + 1e-6).all())
    assert bool(((lse.to(D) - torch.logsumexp(a, 1)).abs() <= lse_bound(Q, K, a)).all())


def test_more_tiles_of_many_rows_than_a_launch_has():
    """4.2 million tiles of 128 rows: 262208 rows of 2056 heads on two keys, of which the last rows, the last heads and some between are looked at."""
    g, rows, n = gen(73), 262208, 2056
    k, v = normal(g, BF16, 2, n, 8), normal(g, BF16, 2, n, 8)
    q, dy = (torch.empty(rows, n, 8, dtype=BF16, device="cuda").normal_(generator=g) for _ in range(2))
    y, lse = B.alpa_attention_forward(q, k, v, scale=0.3, keep_lse=True)
    dq = B.alpa_attention_backward(dy, q, k, v, y, lse, scale=0.3, need=("q",))[0]
    for at, heads in ((slice(0, rows, 4099), slice(0, n)), (slice(rows - 130, rows), slice(0, n)), (slice(0, rows, 97), slice(n - 6, n))):
        Q, E, K, V = q[at, heads].to(D)[:, None], dy[at, heads].to(D)[:, None], k[:, heads].to(D)[None], v[:, heads].to(D)[None]
        a = 0.3 * (Q * K).sum(-1)
        p = torch.softmax(a, 1)[..., None]
        Y = (p * V).sum(1, keepdim=True)
        d = 0.3 * p * ((E * V).sum(-1, keepdim=True) - (E * Y).sum(-1, keepdim=True))
        size = (E * V).abs().sum(-1, keepdim=True) + (E.abs() * V.abs().amax(1, keepdim=True)).sum(-1, keepdim=True)
        assert bool(((y[at, heads].to(D) - Y[:, 0]).abs() <= 4 * 2.0 ** -8 * V.abs().amax(1)).all())
        assert bool(((lse[at, heads].to(D) - torch.logsumexp(a, 1)).abs() <= lse_bound(Q, K, a)).all())
        assert bool(((dq[at, heads].to(D) - (d * K).sum(1)).abs() <= 4 * 2.0 ** -8 * 0.3 * (size * K.abs()).sum(1) + 1e-6).all())
