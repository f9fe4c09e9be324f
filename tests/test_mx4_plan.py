"""The choice of block shapes for MX4 products (mx4_plan.h), compiled with g++: every shape that is
built is taken by some product, alone and grouped by expert. CPU only; test_gpu_mx4.py runs these
products."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (MX4 rows, n, k, m, experts): one product a shape, in their order, for each of fp16 / MX4 rows and
# one matrix / experts
SHAPE_CASES = {
    (0, 0): [(48, 640, 2), (48, 128, 2), (200, 384, 1000), (2050, 128, 100), (100, 1408, 2100), (400, 128, 2100),
             (2050, 128, 700), (4100, 128, 1000), (4100, 128, 2100)],  # not the last shape
    (0, 8): [(48, 640, 2), (48, 128, 2), (100, 640, 1500), (400, 128, 1000), (400, 1408, 700), (1001, 384, 700),
             (2050, 128, 700), (6000, 128, 300), (4100, 128, 2100), (6000, 128, 2)],
    (1, 0): [(48, 1408, 2), (9000, 128, 2), (4100, 384, 50), (4100, 128, 50), (200, 384, 2100), (9000, 384, 50),
             (4100, 1408, 100), (6000, 128, 300), (4100, 128, 1000), (48, 128, 2)],
    (1, 8): [(48, 1408, 2), (4100, 640, 2), (200, 640, 1000), (200, 128, 1500), (400, 1408, 700), (1001, 384, 700),
             (1500, 1408, 300), (2050, 128, 700), (6000, 128, 500), (48, 128, 2)],
}


def shape_cases():
    """(MX4 rows, shape, n, k, m, experts)"""
    return [(a4, i, *c, e) for (a4, e), cs in SHAPE_CASES.items() for i, c in enumerate(cs)]


@pytest.fixture(scope="module")
def pick(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    subprocess.run([gxx, "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
                    os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host", "mx4_plan_model.cpp"), "-o", exe], check=True)

    def run(cases):
        text = "".join("%d %d %d %d %d\n" % c for c in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return run


def test_every_shape_is_taken(pick):
    cases = shape_cases()
    got = pick([(a4, n, k, m, e) for a4, _, n, k, m, e in cases])
    assert [g[0] for g in got] == [c[1] for c in cases]


def test_few_rows_take_small_tiles_and_many_take_large_ones(pick):
    # of experts with a row or none, 32 x 64 measured as good as 16 x 32 with MX4 rows (18.6 and 19.1 us)
    assert all(t[1] <= 32 for t in pick([(a4, 4096, 4096, 16, e) for a4 in (0, 1) for e in (0, 32)]))
    assert all(t[1] >= 128 for t in pick([(a4, 22016, 4096, 4096, e) for a4 in (0, 1) for e in (0, 16)]))


def test_largest_sizes_do_not_overflow(pick):
    big = [(a4, 2**31 - 1, 1 << 20, m, e) for a4 in (0, 1) for m in (1, 65536) for e in (0, 1024)]
    assert all(0 <= t[0] < 10 for t in pick(big))
