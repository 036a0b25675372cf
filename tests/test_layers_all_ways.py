"""Products on every kernel that the library's rule can choose: the rule, asked on the CPU for the sizes of test_layers_ways.py and those here, gives
all of them; the GPU runs these against torch in 64 bits."""
import os
import random
import shutil
import subprocess

import pytest

import test_layers_ways as ways

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# rows, groups, columns of the rows, columns of the result: tiles of 32 x 128 in bf16 fed by the memory unit, whole and in parts; transposed
# products in parts on 256 x 256 tiles; 128 x 128 tiles in parts, and transposed in fp32 through registers
SIZES = [(118, 94, 384, 704), (198, 10, 4032, 2624), (354, 8, 808, 5128), (586, 1, 704, 6272), (1110, 32, 8, 1416), (7790, 109, 167, 1), (269, 5, 672, 488),
         (2142, 125, 232, 88)]
ANY, FED, FEW = 0, 1, 2


def every_kernel():
    """(type, call, kind, tile, in parts) of all that is built."""
    every = set()
    for dtype in ("f32", "bf16"):
        for call in ("y", "dx"):                            # tiles 256 x 256 (bf16, fed), 128 x 128, 64 x 64, 32 x 128
            every |= {(dtype, call, kind, tile, parts) for kind, first in ((FED, dtype == "f32"), (ANY, 1)) for tile in range(first, 4) for parts in (0, 1)}
        every |= {(dtype, "y", FEW, tile, 0) for tile in range(4)}
    every |= {("bf16", "dw", kind, tile, parts) for kind in (FED, ANY) for tile in range(kind == ANY, 3) for parts in (0, 1)}
    every |= {("f32", "dw", kind, tile, parts) for kind in (FED, ANY) for tile, parts in ((0, 0), (1, 0), (1, 1))}
    return every


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    exe, lib = str(tmp_path_factory.mktemp("ways") / "ways_driver"), os.path.join(ROOT, "paper_1902_01064_amd")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(lib, "csrc"),
                    os.path.join(ROOT, "tests", "ways_driver.cpp"), os.path.join(lib, "libhop.so"), "-Wl,-rpath," + lib, "-L/opt/rocm/lib",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True)

    def run(sizes):
        out = subprocess.run([exe], input="".join("%d %d %d %d\n" % s for s in sizes), capture_output=True, text=True, timeout=120, check=True).stdout
        told = [set() for _ in sizes]
        at = -1
        for line in out.splitlines():
            if line == "size":
                at += 1
            else:
                dtype, call, kind, tile, parts = line.split()
                told[at].add((dtype, call, int(kind), int(tile), int(int(parts) > 1)))
        assert at + 1 == len(sizes)
        return told
    return run


def test_the_sizes_take_every_kernel(rule):
    taken = set().union(*rule(ways.SIZES + SIZES))
    assert taken == every_kernel(), (sorted(every_kernel() - taken), sorted(taken - every_kernel()))


def test_no_size_takes_another(rule):
    r = random.Random(1)
    sizes = []
    for _ in range(20000):
        rows, groups, k, n = (int(2 ** r.uniform(0, top)) for top in (18, 12, 14, 14))
        step = r.choice((1, 8, 64))
        sizes.append((rows, groups, -(-k // step) * step, -(-n // step) * step))
    taken = set().union(*rule(sizes))
    assert taken <= every_kernel() and len(taken) > 60


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("size", SIZES)
def test_on_these_sizes(dtype, aligned, size):
    ways.test_every_way(dtype, aligned, size)
