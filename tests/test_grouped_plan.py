"""The choice of block shapes for products of the uniform, codebook and Q4X kinds grouped by expert
(grouped_plan.h), compiled with g++: every shape that is built is taken by some product, of each of the
two sets of costs. CPU only; test_gpu_grouped.py runs these products in every format."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (n, k, m, experts): one product a shape, in their order
SHAPE_CASES = [(33, 384, 3, 3), (33, 128, 3, 3), (1025, 384, 300, 8), (3001, 1408, 300, 8), (1025, 128, 500, 8),
               (3001, 384, 1500, 8)]
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
    assert pick([(bits, kind, *c) for c in SHAPE_CASES]) == [0, 1, 2, 3, 4, 5]


def test_shapes_grow_with_the_rows_of_an_expert(pick):
    for kind in (0, 1):
        rows = [(16, 16, 32, 64, 64, 128)[i] for i in pick([(4, kind, 4096, 2048, 16 * r, 16) for r in (1, 40, 100, 400)])]
        assert rows[0] == 16 and rows == sorted(rows) and rows[2] >= 64 and rows[3] == 128


def test_largest_sizes_do_not_overflow(pick):
    assert all(0 <= t < 6 for t in pick([(4, kind, 2**31 - 1, 1 << 20, m, e) for kind in (0, 1, 2) for m in (1, 65536)
                                         for e in (1, 1024)]))
