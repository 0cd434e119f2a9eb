"""What attention's calls launch, found without a GPU: the library's host code over the HIP runtime that tests/fake_layers_driver.cpp makes up
(tests/fake_blocks_driver.cpp has the calls)."""
import os
import re
import subprocess
from collections import namedtuple

from paper_2201_12023_amd import binding as B
from tests.layer_launches import ROOT, TYPES, calls                # noqa: F401

# kind: y, y_few, dq, dq_few, dkv; blocks: of 32 elements of a head; score: plain, extra (capped or biased), far (a cap above 256); detail: (waves, dk, dv) of dkv
Kernel = namedtuple("Kernel", "kind type blocks score detail")
Launch = namedtuple("Launch", "kernel grid splits")
KINDS = {"attention_kernel": "y", "attention_few_kernel": "y_few", "attention_dq_kernel": "dq", "attention_dq_few_kernel": "dq_few", "attention_dkv_kernel": "dkv"}


def build(folder):
    out = os.path.join(str(folder), "blocks_driver")
    # (the library's other imports are the real runtime's, which is loaded and never called)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused-function", "-rdynamic", "-o", out, os.path.join(ROOT, "tests", "fake_blocks_driver.cpp"),
                           B.LIB_PATH, "-Wl,--allow-shlib-undefined"])
    return out


def launches(call):
    """Attention's launches among a call's, in their order; joins as kinds join_y, join_dq (splits: packed rows of a tile) and sum."""
    out = []
    for name, x, y, _, _ in call.launches:
        m = re.match(r"_ZN4alpa\d+(attention\w*?_kernel)I(f|DF16_|DF16b)(.*?)EEv", name)
        if not m:
            continue
        kind, kind_of, rest = KINDS.get(m.group(1)), TYPES[m.group(2)], re.findall(r"L[ib](\d+)E", m.group(3) + "E")
        if kind is None:
            join = m.group(1) == "attention_join_kernel"
            out.append(Launch(Kernel(("join_dq" if rest[0] == "1" else "join_y") if join else "sum", kind_of, 0, "", None), x, 8 * y if join else y))
            continue
        blocks, extra, far = int(rest[0]), rest[1] == "1", rest[-1] == "1"
        detail = (int(rest[2]), rest[3] == "1", rest[4] == "1") if kind == "dkv" else None
        out.append(Launch(Kernel(kind, kind_of, blocks, "far" if far else "extra" if extra else "plain", detail), x, y))
    return out
