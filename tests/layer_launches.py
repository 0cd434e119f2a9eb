"""What the layer operators' calls launch, found without a GPU: the library's host code over the HIP runtime that
tests/fake_layers_driver.cpp makes up."""
import os
import re
import subprocess
from collections import namedtuple

from paper_2201_12023_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
Call = namedtuple("Call", "rc work launches")                       # launches: (kernel, grid x, y, z, threads)
Product = namedtuple("Product", "type a b tile epilogue grouping grid splits")
TYPES = {"f": "f32", "DF16_": "f16", "DF16b": "bf16"}
FORMS, EPILOGUES, GROUPINGS = ("ROWS", "COLS"), ("LINE", "SIGMOID", "ERF", "SUM", "LOSS", "GRAD"), ("NONE", "ROWS", "STEPS")


def build(folder):
    out = os.path.join(str(folder), "layers_driver")
    # (the library's other imports are the real runtime's, which is loaded and never called)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-rdynamic", "-o", out, os.path.join(ROOT, "tests", "fake_layers_driver.cpp"),
                           B.LIB_PATH, "-Wl,--allow-shlib-undefined"])
    return out


def calls(driver, lines):
    """One Call for each line (see the driver)."""
    env = dict(os.environ)
    env["LD_LIBRARY_PATH"] = os.path.dirname(B.LIB_PATH) + ":" + env.get("LD_LIBRARY_PATH", "")
    text = "".join(" ".join(str(int(v)) if not isinstance(v, str) else v for v in line) + "\n" for line in lines)
    r = subprocess.run([driver], input=text, stdout=subprocess.PIPE, text=True, env=env, timeout=120, check=True)
    out = []
    for line in r.stdout.splitlines():
        head, *rest = line.split(" ", 2)
        work, launches = rest[0], rest[1] if len(rest) > 1 else ""
        found = [part.split() for part in launches.split(";") if part.strip()]
        out.append(Call(int(head), int(work), [(f[0], *map(int, f[1:])) for f in found]))
    assert len(out) == len(lines)
    return out


def products(call):
    """The products among a call's launches, in their order."""
    out = []
    for name, x, y, _, _ in call.launches:
        m = re.search(r"product_kernelI(f|DF16_|DF16b)Li(\d)ELi(\d)ELi(\d+)ELi\d+ELi\d+ELi\d+ELi(\d)ELi(\d)E", name)
        if m:
            t, a, b, tile, epi, grouping = m.groups()
            out.append(Product(TYPES[t], FORMS[int(a)], FORMS[int(b)], int(tile), EPILOGUES[int(epi)], GROUPINGS[int(grouping)], x, y))
    return out
