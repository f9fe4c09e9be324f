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
    (0, 0): [(48, 384, 2), (48, 128, 2), (200, 384, 1000), (200, 128, 1500), (200, 896, 1500), (6000, 128, 100),
             (2050, 128, 500), (4100, 128, 700), (4100, 128, 2100)],
    (0, 8): [(48, 384, 2), (48, 128, 2), (200, 384, 1000), (200, 128, 1500), (200, 896, 1500), (400, 128, 1500),
             (3000, 128, 200), (6000, 128, 100), (6000, 128, 1000)],
    (1, 0): [(48, 896, 2), (48, 128, 2), (100, 384, 2100), (200, 128, 1500), (3000, 2176, 100), (2050, 896, 500),
             (1001, 896, 1000), (4100, 128, 700), (4100, 128, 1500)],
    (1, 8): [(48, 896, 2), (48, 128, 2), (100, 384, 2100), (3000, 128, 9), (1500, 2176, 200), (400, 1408, 2100),
             (400, 1408, 2100), (3000, 128, 700), (4100, 128, 1000)],
}
EXPERTS = {(0, 8): [3, 3, 3, 3, 3, 8, 8, 8, 8], (1, 8): [3, 3, 3, 8, 3, 8, 3, 8, 8]}


def shape_cases():
    """(MX4 rows, shape, n, k, m, experts)"""
    return [(a4, i, *c, EXPERTS[a4, e][i] if e else 0) for (a4, e), cs in SHAPE_CASES.items() for i, c in enumerate(cs)]


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
    assert all(0 <= t[0] < 9 for t in pick(big))
