"""Shapes that reach each of attention's compiled kernels: rows in tiles of 128 or few, keys or rows in one part or several, keys of the gradients in tiles of 128 and 256, and
the few rows of a sequence a workgroup, among them one of many.

That the shapes reach what they are listed for is checked without a GPU (tests/test_blocks_host_side.py), so a change of the rules is noticed there;
tests/test_gpu_blocks_paths.py runs them, each with heads of every number of blocks of 32 elements, and with scores as they are, capped and biased, and under a cap far above."""
from collections import namedtuple

DIMS = {2: 40, 3: 96, 4: 104, 8: 200}                # blocks as compiled: elements
CAPS = {"plain": 0.0, "extra": 6.0, "far": 1000.0}

# y, dq, dkv: kind and parts (1, or 2 for several) in 16 bits, and in 32 where they differ; tile: keys of a workgroup of dkv in 16 bits, heads up to 128
Shape = namedtuple("Shape", "rows k_rows heads kv_heads lens k_lens causal prefix y dq dkv tile wide")
MANY, FEW = ("y", "dq"), ("y_few", "dq_few")
SHAPES = {
    "many rows": Shape(1100, 1300, 32, 16, (600, 480), (700, 590), True, (300, 0), ("y", 1), ("dq", 1), 2, 128, {}),
    "many rows, keys in parts": Shape(4150, 4200, 8, 8, (4150,), (4200,), True, (40,), ("y", 2), ("dq", 2), 2, 256, {"dq": ("dq", 1)}),
    "many rows, rows in one part": Shape(1100, 1300, 64, 64, (500, 0, 590), (700, 30, 500), False, None, ("y", 1), ("dq", 1), 1, 128, {}),
    "many keys, rows in one part": Shape(400, 1300, 32, 32, (250, 140), (620, 650), False, None, ("y_few", 1), ("dq_few", 1), 1, 256, {}),
    "few rows": Shape(150, 60, 4, 2, (150,), (60,), True, (7,), ("y_few", 1), ("dq_few", 1), 2, 128, {}),
    "few rows, keys in parts": Shape(150, 700, 4, 2, (150,), (700,), True, None, ("y_few", 2), ("dq_few", 2), 2, 128, {}),
    # (one sequence has six tiles of 32 packed rows, one after the other in a workgroup of y)
    "one long sequence among short ones": Shape(102, 1060, 4, 2, (90, 1, 2, 0, 1, 3, 2, 1), (300, 17, 500, 40, 0, 3, 129, 64), True, (0, 0, 9, 0, 5, 1, 200, 0),
                                               ("y_few", 1), ("dq_few", 1), 1, 128, {"y": ("y_few", 2), "dq": ("dq_few", 2)}),
    "one long sequence among short ones, keys in parts": Shape(102, 4010, 4, 2, (90, 1, 2, 0, 1, 3, 2, 1), (1300, 170, 1500, 400, 0, 3, 529, 64), True, None,
                                                               ("y_few", 2), ("dq_few", 2), 1, 128, {}),
}


def line(back, dtype, shape, dim, score):
    """A call as tests/fake_blocks_driver.cpp reads it."""
    return ("attention", back, dtype, len(shape.lens), shape.heads, shape.kv_heads, dim, shape.causal, 1, shape.rows, shape.k_rows, str(CAPS[score]), score != "plain", 7)
