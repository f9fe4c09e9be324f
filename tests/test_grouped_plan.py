"""The choice of block shapes for products of the uniform, codebook and Q4X kinds grouped by expert
(grouped_plan.h), compiled with g++: every shape that is built is taken by some product, of each of the
two sets of costs. CPU only; test_gpu_grouped.py runs these products in every format."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (n, k, m, experts): one product a shape, in their order
SHAPE_CASES = [(33, 384, 3, 3), (513, 128, 700, 3), (1025, 128, 700, 8), (3001, 128, 700, 8), (3001, 640, 1500, 8)]
FORMATS = [(b, kind, g) for b in (3, 4) for kind in (0, 1) for g in (32, 64, 128)] + [(4, 2, 64)]


@pytest.fixture(scope="module")
def pick(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    subprocess.run([gxx, "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
                    os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host", "grouped_plan_model.cpp"), "-o", exe],
                   check=True)

    def run(cases):
        text = "".join("%d %d %d %d %d %d\n" % c for c in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60).stdout
        return [int(v) for v in out.split()]
    return run


@pytest.mark.parametrize("bits,kind", sorted({f[:2] for f in FORMATS}))
def test_every_shape_is_taken(pick, bits, kind):
    assert pick([(bits, kind, *c) for c in SHAPE_CASES]) == [0, 1, 2, 3, 4]


def test_shapes_grow_with_the_rows_of_an_expert(pick):
    for kind in (0, 1):
        got = pick([(4, kind, 4096, 2048, m, 16) for m in (16, 16 * 24, 16 * 400)])
        assert got[0] == 0 and got[1] == 1 and got[2] == 4


def test_largest_sizes_do_not_overflow(pick):
    assert all(0 <= t < 5 for t in pick([(4, kind, 2**31 - 1, 1 << 20, m, e) for kind in (0, 1, 2) for m in (1, 65536)
                                         for e in (1, 1024)]))
