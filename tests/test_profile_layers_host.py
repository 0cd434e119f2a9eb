"""The options that profile_layers makes from measured times: no GPU, the times are given."""
import numpy as np
import pytest

from paper_2201_12023_amd import profile_layers as P
from paper_2201_12023_amd import workloads as W

MODEL = P.Model(layers=4, rows=24, width=8, inner=16, experts=2, expert_every=2, words=64)


def given(share):
    return np.array([1000.0 * (k + 1) * share.rows * share.inner / 384 for k in range(share.layers)])


def test_kinds_weights_and_shares():
    assert [MODEL.kind(k) for k in range(4)] == ["dense", "experts", "dense", "experts"]
    dense = 2 * 8 * 16 + 16 + 8
    assert [MODEL.weights(k) for k in range(4)] == [dense, 2 * dense, dense, 2 * dense + 64 * 8]
    assert MODEL.share(8, "rows").rows == 3 and MODEL.share(8, "rows").inner == 16
    assert MODEL.share(8, "weights").inner == 2 and MODEL.share(8, "weights").words == 8
    assert MODEL.share(16, "rows") is None and MODEL.share(32, "weights") is None


def test_options_of_every_stage_and_submesh():
    shapes = W.submesh_shapes(2, 8)
    asked = []
    t_l, stage, act = P.profiles(MODEL, shapes, 4, 2e6, lambda m: asked.append(m) or given(m))
    assert t_l.shape == stage.shape == act.shape == (4, 4, len(shapes), 2)
    assert len(asked) == len(set(asked))                         # one device: both options are one share
    for q, (n, m) in enumerate(shapes):
        d = int(n * m)
        for o, split in enumerate(P.SPLITS):
            share = MODEL.share(d, split)
            if share is None:
                assert (t_l[:, :, q, o] == P.INF).all()
                continue
            for k in range(4):
                for i in range(k, 4):
                    sent = [2 * (MODEL.weights(j) / 4 if o == 0 else 2 * 24 * 8) * 2 * (d - 1) / d / 2.0 for j in range(k, i + 1)]
                    assert abs(int(t_l[k, i, q, o]) - sum(given(share)[k:i + 1]) - sum(sent)) <= 1.001
                    assert stage[k, i, q, o] == 16 * sum(share.weights(j) for j in range(k, i + 1))
                    assert act[k, i, q, o] == 2 * share.rows * (8 + 2 * share.inner) * (i - k + 1)
    assert (t_l[np.tril_indices(4, -1)] == P.INF).all()          # no stage ends before it begins


def test_sizes_from_the_command_line_are_checked():
    with pytest.raises(SystemExit):
        P.main(["--layers", "many"])
