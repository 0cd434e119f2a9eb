"""The options of blocks with attention: no GPU, the times are given."""
import numpy as np

from paper_2201_12023_amd import profile_layers as P
from paper_2201_12023_amd import workloads as W

MODEL = P.Model(layers=2, rows=32, width=8, inner=16, experts=2, expert_every=0, words=64, heads=4, kv_heads=2, dim=6, context=8)


def test_weights_and_shares():
    products, attention = 2 * 8 * 16 + 16 + 8, 8 * (4 + 2 * 2) * 6 + 4 * 6 * 8 + 4 * 8
    assert [MODEL.weights(k) for k in range(2)] == [products + attention, products + attention + 64 * 8]
    share = MODEL.share(2, "weights")
    assert (share.heads, share.kv, share.dim, share.inner, share.words, share.rows) == (2, 1, 6, 8, 32, 32)
    assert MODEL.share(4, "weights") is None                      # (two kv heads)
    assert MODEL.share(4, "rows").rows == 8 and MODEL.share(8, "rows") is None         # (sequences of eight rows stay whole)
    assert MODEL.share(1, "rows").rows == 32 and MODEL.share(1, "weights").kv == 2
    alone = P.Model(heads=4)
    assert alone.kv == 4 and alone.share(4, "weights").heads == 1 and P.Model().share(8, "rows").rows == 512


def test_options():
    shapes = W.submesh_shapes(1, 4)
    t_l, stage, act = P.profiles(MODEL, shapes, 4, 2e6, lambda m: np.array([1000.0, 2000.0]))
    for q, (n, m) in enumerate(shapes):
        d = int(n * m)
        for o, split in enumerate(P.SPLITS):
            share = MODEL.share(d, split)
            if share is None:
                assert (t_l[:, :, q, o] == P.INF).all()
                continue
            sent = [2 * (MODEL.weights(k) / 4 if o == 0 else 4 * 32 * 8) * 2 * (d - 1) / d / 2.0 for k in range(2)]
            assert abs(int(t_l[0, 1, q, o]) - 3000.0 - sum(sent)) <= 1.001
            assert stage[0, 1, q, o] == 16 * (share.weights(0) + share.weights(1))
            floats = share.rows * (share.heads + 4)
            halves = share.rows * (4 * 8 + 2 * share.inner + 2 * (share.heads + share.kv) * 6)
            assert act[0, 0, q, o] == 2 * halves + 4 * floats
