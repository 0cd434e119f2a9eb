"""Sizes that reach each of the compiled products: tile, forms of the operands, epilogue, grouping, and the contraction split or not.

A large tile's workgroups take two tiles and more where the contraction is not split, some of them; sizes end inside tiles.  That the sizes
reach what they are listed for is checked without a GPU (tests/test_layers_host_side.py), so a change of how products are cut is noticed there;
tests/test_gpu_layers_paths.py runs them."""

# path: (first operand, second, tile, epilogue, grouping, split); then the call in 16 bits and in 32: (name, act, rows, experts, n_in, n_out)
PATHS = [
    (("COLS", "COLS", 256, "LINE", "NONE", False), ("backward", 3, 207, -1, 8768, 2832), ("gradient", 0, 229, -1, 8104, 3832)),
    (("COLS", "COLS", 128, "LINE", "NONE", False), ("gradient", 0, 71, -1, 7528, 272), ("gradient", 0, 71, -1, 6540, 320)),
    (("COLS", "COLS", 64, "LINE", "NONE", False), ("gradient", 0, 73, -1, 8, 8), ("gradient", 0, 73, -1, 8, 8)),
    (("COLS", "COLS", 256, "SUM", "NONE", True), ("gradient", 0, 8925, -1, 5936, 152), ("backward", 0, 1853, -1, 3528, 1432)),
    (("COLS", "COLS", 128, "SUM", "NONE", True), ("gradient", 0, 9523, -1, 2896, 80), ("gradient", 0, 747, -1, 80, 8600)),
    (("COLS", "COLS", 64, "SUM", "NONE", True), ("gradient", 0, 1793, -1, 8, 8), ("gradient", 0, 547, -1, 8, 8)),
    (("COLS", "COLS", 256, "LINE", "STEPS", False), ("backward", 0, 1255, 6, 6648, 541), ("backward", 3, 3727, 16, 432, 3992)),
    (("COLS", "COLS", 128, "LINE", "STEPS", False), ("backward", 3, 1437, 19, 8, 5240), ("backward", 3, 1661, 18, 1840, 72)),
    (("COLS", "COLS", 64, "LINE", "STEPS", False), ("backward", 2, 231, 2, 16, 8), ("backward", 0, 219, 3, 8, 8)),
    (("ROWS", "COLS", 256, "LINE", "NONE", False), ("backward", 2, 28479, -1, 792, 200), ("gradient", 0, 6553, -1, 4384, 232)),
    (("ROWS", "COLS", 128, "LINE", "NONE", False), ("gradient", 0, 35115, -1, 8, 80), ("backward", 3, 12123, -1, 136, 72)),
    (("ROWS", "COLS", 64, "LINE", "NONE", False), ("backward", 0, 1, -1, 8, 72), ("backward", 3, 1, -1, 8, 72)),
    (("ROWS", "COLS", 256, "SUM", "NONE", False), ("gradient", 0, 26263, -1, 872, 5440), ("gradient", 0, 29551, -1, 1440, 2240)),
    (("ROWS", "COLS", 128, "SUM", "NONE", False), ("gradient", 0, 39623, -1, 66, 3352), ("gradient", 0, 30953, -1, 80, 2083)),
    (("ROWS", "COLS", 64, "SUM", "NONE", False), ("gradient", 0, 23621, -1, 8, 5816), ("gradient", 0, 34811, -1, 8, 1832)),
    (("ROWS", "COLS", 256, "SUM", "NONE", True), ("backward", 2, 5765, -1, 144, 8032), ("gradient", 0, 20741, -1, 216, 1928)),
    (("ROWS", "COLS", 128, "SUM", "NONE", True), ("gradient", 0, 67, -1, 4376, 7656), ("gradient", 0, 8303, -1, 72, 922)),
    (("ROWS", "COLS", 64, "SUM", "NONE", True), ("gradient", 0, 1, -1, 8, 1872), ("gradient", 0, 1, -1, 8, 544)),
    (("ROWS", "COLS", 256, "LINE", "ROWS", False), ("backward", 2, 5149, 23, 3912, 272), ("backward", 2, 4385, 5, 6632, 288)),
    (("ROWS", "COLS", 128, "LINE", "ROWS", False), ("backward", 3, 29, 12, 6608, 88), ("backward", 0, 121, 9, 5712, 80)),
    (("ROWS", "COLS", 64, "LINE", "ROWS", False), ("backward", 0, 7, 2, 8, 112), ("backward", 3, 5, 2, 8, 120)),
    (("ROWS", "ROWS", 256, "ERF", "NONE", False), ("forward", 2, 32109, -1, 245, 808), ("forward", 2, 13397, -1, 272, 3568)),
    (("ROWS", "ROWS", 128, "ERF", "NONE", False), ("forward", 2, 10969, -1, 72, 136), ("forward", 2, 18391, -1, 88, 107)),
    (("ROWS", "ROWS", 64, "ERF", "NONE", False), ("forward", 2, 1, -1, 96, 8), ("forward", 2, 1, -1, 72, 8)),
    (("ROWS", "ROWS", 256, "GRAD", "NONE", False), ("gradient", 0, 8055, -1, 208, 3152), ("gradient", 0, 7899, -1, 208, 3896)),
    (("ROWS", "ROWS", 128, "GRAD", "NONE", False), ("gradient", 0, 33903, -1, 76, 8), ("gradient", 0, 17651, -1, 96, 80)),
    (("ROWS", "ROWS", 64, "GRAD", "NONE", False), ("gradient", 0, 1, -1, 72, 8), ("gradient", 0, 1, -1, 72, 8)),
    (("ROWS", "ROWS", 256, "LINE", "NONE", False), ("forward", 0, 16895, -1, 216, 1928), ("forward", 0, 14541, -1, 240, 3208)),
    (("ROWS", "ROWS", 128, "LINE", "NONE", False), ("forward", 0, 34585, -1, 112, 8), ("forward", 0, 281, -1, 72, 6690)),
    (("ROWS", "ROWS", 64, "LINE", "NONE", False), ("forward", 0, 1, -1, 80, 8), ("forward", 0, 1, -1, 120, 8)),
    (("ROWS", "ROWS", 256, "LOSS", "NONE", False), ("loss", 0, 33849, -1, 200, 656), ("loss", 0, 12619, -1, 208, 2392)),
    (("ROWS", "ROWS", 128, "LOSS", "NONE", False), ("loss", 0, 34207, -1, 88, 8), ("loss", 0, 8199, -1, 80, 200)),
    (("ROWS", "ROWS", 64, "LOSS", "NONE", False), ("loss", 0, 1, -1, 72, 8), ("loss", 0, 1, -1, 80, 8)),
    (("ROWS", "ROWS", 256, "SIGMOID", "NONE", False), ("forward", 3, 9421, -1, 264, 4128), ("forward", 3, 13321, -1, 248, 2280)),
    (("ROWS", "ROWS", 128, "SIGMOID", "NONE", False), ("forward", 3, 38157, -1, 120, 8), ("forward", 3, 13281, -1, 72, 152)),
    (("ROWS", "ROWS", 64, "SIGMOID", "NONE", False), ("forward", 3, 1, -1, 88, 16), ("forward", 3, 1, -1, 96, 8)),
    (("ROWS", "ROWS", 256, "SUM", "NONE", True), ("forward", 2, 10981, -1, 5048, 160), ("forward", 0, 1239, -1, 1336, 4288)),
    (("ROWS", "ROWS", 128, "SUM", "NONE", True), ("forward", 2, 69, -1, 8624, 3296), ("forward", 0, 77, -1, 2808, 3264)),
    (("ROWS", "ROWS", 64, "SUM", "NONE", True), ("forward", 0, 1, -1, 1928, 8), ("forward", 2, 1, -1, 536, 8)),
    (("ROWS", "ROWS", 256, "ERF", "ROWS", False), ("forward", 2, 16503, 4, 216, 1984), ("forward", 2, 19861, 6, 232, 1528)),
    (("ROWS", "ROWS", 128, "ERF", "ROWS", False), ("forward", 2, 34237, 18, 80, 16), ("forward", 2, 59, 5, 96, 9704)),
    (("ROWS", "ROWS", 64, "ERF", "ROWS", False), ("forward", 2, 13, 3, 104, 8), ("forward", 2, 9, 4, 88, 8)),
    (("ROWS", "ROWS", 256, "LINE", "ROWS", False), ("forward", 0, 36071, 4, 200, 1016), ("forward", 0, 29759, 18, 216, 1000)),
    (("ROWS", "ROWS", 128, "LINE", "ROWS", False), ("forward", 0, 33163, 2, 77, 8), ("forward", 0, 541, 5, 76, 4464)),
    (("ROWS", "ROWS", 64, "LINE", "ROWS", False), ("forward", 0, 13, 3, 72, 8), ("forward", 0, 5, 2, 112, 8)),
    (("ROWS", "ROWS", 256, "SIGMOID", "ROWS", False), ("forward", 3, 4037, 8, 232, 6360), ("forward", 3, 16207, 19, 1048, 1784)),
    (("ROWS", "ROWS", 128, "SIGMOID", "ROWS", False), ("forward", 3, 36285, 5, 80, 8), ("forward", 3, 125, 7, 80, 11992)),
    (("ROWS", "ROWS", 64, "SIGMOID", "ROWS", False), ("forward", 3, 15, 3, 121, 8), ("forward", 3, 5, 2, 144, 8)),
]


def line(dtype, case):
    """A case as tests/layer_launches.py takes it."""
    name, act, rows, experts, n_in, n_out = case
    if name == "forward":
        return name, dtype, act, rows, experts, n_in, n_out, n_in, n_out, 1, 1, 1
    if name == "backward":
        return name, dtype, act, rows, experts, n_in, n_out, n_in, n_in, 1, 1, 1
    return name, dtype, rows, n_in, n_out
