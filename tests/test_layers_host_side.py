"""What the layer operators' calls queue and ask for, looked at without a GPU (tests/layer_launches.py)."""
import shutil

import pytest

from tests import layer_launches as Q
from tests import layer_paths as P

F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++ here")
    return Q.build(tmp_path_factory.mktemp("layers"))


@pytest.mark.parametrize("rows", [(1 << 26) - 16, (1 << 26) - 15, 1 << 26, (1 << 27) + 1, 1 << 28])
def test_loss_of_many_rows_is_launched(driver, rows):
    """As many rows as the header allows; HIP counts a grid's threads in 32 bits, and a loss takes 64 a row."""
    call, = Q.calls(driver, [("loss", BF16, rows, 8, 64)])
    assert call.rc == 0 and "loss_kernel" in call.launches[-1][0]
    assert call.launches[-1][1] == min((rows + 15) // 16, 1 << 21)


@pytest.mark.parametrize("line", [("backward", BF16, 0, 809, 3357, 922983, 7, 922983, 922983, 0, 1, 1),
                                  ("backward", BF16, 0, 1500, 4096, 300000, 1, 300000, 300000, 0, 0, 1),
                                  ("forward", BF16, 0, 4096, 4096, 8, 1 << 20, 8, 1 << 20, 0, 0, 0)])
def test_products_of_many_tiles_are_launched(driver, line):
    """Weights of 4096 experts make more tiles than one launch has threads for: every tile is in one of the launches."""
    call, = Q.calls(driver, [line])
    assert call.rc == 0
    _, _, _, rows, experts, n_in, n_out = line[:7]
    for p in Q.products(call):
        assert p.grid <= 1 << 23
    steps = [p for p in Q.products(call) if p.grouping == "STEPS"]
    if steps and steps[0].tile < 256:
        t = steps[0].tile
        assert sum(p.grid for p in steps) == -(-(-(-n_out // t) * -(-n_in // t)) // 8) * 8 * experts


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("rows, words", [(1, 5), (65536, 1024), (65537, 5000), (131072, 51200), (131073, 1024), (200000, 51200), (1 << 20, 2),
                                         (1 << 24, 1030)])
def test_work_memory_of_the_loss_backwards(driver, dtype, rows, words):
    """The gradient of the logits is in memory 256 MiB at a time, whatever the number of rows; beside it stand a float a row, the
    32-bit sums of dx and of a piece's dw, and the parts of products that are split (2^26 floats at most)."""
    n_in = 8
    call, = Q.calls(driver, [("gradient", dtype, rows, n_in, words)])
    assert call.rc == 0
    assert call.work <= (256 << 20) + rows * 4 + rows * n_in * 4 + words * n_in * 4 + (1 << 28) + (1 << 14)
    pieces = [p for p in Q.products(call) if p.epilogue == "GRAD"]
    assert len(pieces) >= rows * words * (4 if dtype == F32 else 2) / (256 << 20)


def test_listed_sizes_reach_every_product(driver):
    """Each of tests/layer_paths.py's cases takes the path that it is listed for, and no compiled product is left without one."""
    seen = set()
    for dtype in (F32, F16, BF16):
        cases = [small if dtype != F32 else wide for _, small, wide in P.PATHS]
        for (path, _, _), case, call in zip(P.PATHS, cases, Q.calls(driver, [P.line(dtype, c) for c in cases])):
            assert call.rc == 0
            found = {(p.a, p.b, p.tile, p.epilogue, p.grouping, p.splits > 1): p for p in Q.products(call)}
            assert path in found, (path, case)
            p = found[path]
            assert path[2] < 256 or path[5] or p.grid == 256
            seen.add((p.type, *path[:5]))
    # sums over blocks of rows without parts (tests/test_gpu_layers_edges.py)
    for call in Q.calls(driver, [("gradient", BF16, 131072 + 28, 16376, 1000), ("gradient", F32, 65536 + 28, 16376, 1000)]):
        assert [(p.tile, p.splits) for p in Q.products(call) if p.epilogue == "SUM"] == [(256, 1)] * 2
    there, = Q.calls(driver, [("kernels",)])
    assert seen == {(p.type, p.a, p.b, p.tile, p.epilogue, p.grouping) for p in Q.products(there)} and len(seen) == 135


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_results_that_are_not_aligned_take_a_smaller_tile(driver, dtype):
    """The sizes of tests/test_gpu_layers_bounds.py, with rows of the result as long as they are apart, and three elements further."""
    dense, experts = (9000, -1, 5128, 5128), (131 * 96, 4, 2568, 3592)
    tiles = []
    for pad in (0, 3):
        lines = [("forward", dtype, 3, *s, s[2], s[3] + pad, 1, 1, 1) for s in (dense, experts)]
        lines.append(("backward", dtype, 3, *dense, dense[2], dense[2] + pad, 1, 1, 0))
        tiles.append([Q.products(call)[0].tile for call in Q.calls(driver, lines)])
    assert tiles == [[256] * 3, [128] * 3]


@pytest.mark.parametrize("dtype, rows, n_in, words", [(BF16, 200000, 1024, 32000), (BF16, 600000, 512, 1024), (F32, 140000, 24, 1024)])
def test_gradients_of_blocks_of_rows_fill_the_compute_units(driver, dtype, rows, n_in, words):
    """Rows in blocks: a piece's dw has few tiles and a long contraction, which is split as it is without blocks, and joined to the blocks before."""
    call, = Q.calls(driver, [("gradient", dtype, rows, n_in, words)])
    assert call.rc == 0
    dw = [p for p in Q.products(call) if (p.a, p.b) == ("COLS", "COLS")]
    grads = [p for p in Q.products(call) if p.epilogue == "GRAD"]
    assert len(dw) == len(grads) and all(p.splits > 1 for p in dw)
    assert sum("join_kernel" in name for name, *_ in call.launches) >= len(dw)
