"""What attention's calls queue, looked at without a GPU (tests/block_launches.py)."""
import shutil

import pytest

from tests import block_launches as Q
from tests import block_paths as P

F32, F16, BF16 = 0, 1, 2
NAMES = {F32: "f32", F16: "f16", BF16: "bf16"}


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++ here")
    return Q.build(tmp_path_factory.mktemp("blocks"))


def expected(shape, dtype, blocks, score):
    """The kernels of a forward and a backward call, each with whether its launch is in parts, joins among them."""
    t, parts = NAMES[dtype], lambda n: n > 1
    score = "extra" if score == "far" and dtype == F32 else score
    pick = lambda name: shape.wide.get(name, getattr(shape, name)) if dtype == F32 else getattr(shape, name)
    (y, y_parts), (dq, dq_parts) = pick("y"), pick("dq")
    forward = {Q.Kernel(y, t, blocks, score, None): parts(y_parts)}
    if parts(y_parts):
        forward[Q.Kernel("join_y", t, 0, "", None)] = 32 if y == "y_few" else 128
    back = {Q.Kernel(dq, t, blocks, score, None): parts(dq_parts)}
    if parts(dq_parts):
        back[Q.Kernel("join_dq", t, 0, "", None)] = 32 if dq == "dq_few" else 128
    waves = shape.tile // 32 if dtype != F32 and blocks < 8 else 4
    for detail in ((waves, True, True),) if blocks < 8 else ((4, True, False), (4, False, True)):
        back[Q.Kernel("dkv", t, blocks, score, detail)] = parts(shape.dkv)
    if parts(shape.dkv):
        back[Q.Kernel("sum", t, 0, "", None)] = None
    return forward, back


def test_listed_shapes_reach_every_kernel(driver):
    """Each of tests/block_paths.py's shapes takes the path that it is listed for, and no compiled kernel of attention is left without one, in one part and (but for
    those that never go in parts) in several."""
    seen = set()
    for dtype in (F32, F16, BF16):
        for name, shape in P.SHAPES.items():
            assert sum(shape.lens) <= shape.rows and sum(shape.k_lens) <= shape.k_rows
            for blocks, dim in P.DIMS.items():
                for score in P.CAPS:
                    calls = Q.calls(driver, [P.line(back, dtype, shape, dim, score) for back in (0, 1)])
                    for call, want in zip(calls, expected(shape, dtype, blocks, score)):
                        assert call.rc == 0
                        got = {s.kernel: s.splits for s in Q.launches(call)}
                        for k, v in got.items():
                            joins = k.kind in ("join_y", "join_dq")
                            if k in want:
                                assert joins and v == want[k] or k.kind == "sum" or (not joins and (v > 1) == want[k]), (name, k, v)
                            seen.add((k, v if joins else v > 1 if k.kind != "sum" else None))
                        assert set(got) == set(want), (name, NAMES[dtype], blocks, score)
    there, = Q.calls(driver, [("kernels",)])
    compiled = {s.kernel for s in Q.launches(there)}
    assert {k for k, _ in seen} == compiled and len(compiled) == 195
    lacking = set()
    for k in compiled:
        if k.kind in ("join_y", "join_dq"):
            lacking |= {(k, n) for n in (32, 128)} - seen
        elif k.kind != "sum":
            lacking |= {(k, False), (k, True)} - seen
    # dq of many rows in 32 bits never goes in parts
    assert {(k.kind, k.type, n) for k, n in lacking} == {("dq", "f32", True), ("join_dq", "f32", 128)}, lacking


def test_more_workgroups_than_a_launch_has(driver):
    """2^22 workgroups a launch at most, HIP counting a grid's threads in 32 bits: the others go in further launches, all of them in some."""
    for dtype, seqs, n, rows, k_rows in ((BF16, 1030, 4096, 1030, 2060), (BF16, 1, 2056, 262208, 2), (F32, 65536, 65, 65536, 65536)):
        for back, kinds in ((0, {"y", "y_few"}), (1, {"dq", "dq_few"}), (1, {"dkv"})):
            call, = Q.calls(driver, [("attention", back, dtype, seqs, n, n, 8, 0, 1, rows, k_rows, "0", 0, 7)])
            assert call.rc == 0
            found = [s for s in Q.launches(call) if s.kernel.kind in kinds]
            tile = {"y": 128, "dq": 128, "dq_few": 32, "y_few": 0, "dkv": 128}[found[0].kernel.kind]
            packed = k_rows if "dkv" in kinds else rows
            tiles = (seqs + 1) if tile == 0 else packed // tile + min(seqs + 2, packed)
            assert [s.grid for s in found[:-1]] == [1 << 22] * (len(found) - 1) and sum(s.grid for s in found) == tiles * n and all(s.splits == 1 for s in found)
            assert len(found) > 1 or k_rows == 2 and back
