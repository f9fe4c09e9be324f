"""Products that take every block shape of the MX4 and the grouped tiles through several stages: buffers are
loaded again, rows of scales begin anew, and the last stage is moved back to the end of the row. The choice
of shapes is compiled with g++ (CPU only); test_gpu_stages.py runs the products."""
import os
import shutil
import subprocess

import pytest

from test_grouped_plan import FORMATS, ROOT

# (MX4 rows, experts): (shape, n, k, m)
MX4_CASES = {
    (0, 0): [(0, 33, 2176, 3), (0, 33, 5248, 3), (1, 33, 1152, 1501), (1, 33, 1920, 1501), (2, 33, 1152, 3001),
             (2, 33, 1920, 3001), (3, 77, 640, 3001), (3, 33, 384, 4097), (3, 4101, 1408, 77), (4, 33, 1920, 4097),
             (5, 131, 640, 4097), (5, 13001, 384, 33), (5, 131, 1408, 4097), (6, 1501, 640, 1001), (6, 3001, 1280, 523), (6, 1001, 384, 1501),
             (7, 1501, 640, 3001), (7, 1001, 384, 4097), (8, 2051, 640, 4097), (8, 2051, 384, 4097)],
    (0, 8): [(0, 33, 2176, 2), (0, 33, 5248, 2), (1, 33, 1152, 1501), (1, 33, 1920, 1501), (2, 33, 1152, 3001),
             (2, 33, 1920, 3001), (3, 77, 640, 3001), (3, 131, 384, 2101), (3, 523, 1408, 701), (4, 77, 1152, 3001),
             (4, 77, 1920, 3001), (5, 131, 640, 4097), (5, 131, 384, 4097), (5, 131, 1408, 4097), (6, 701, 640, 2101),
             (6, 2051, 1280, 701), (6, 701, 384, 2101), (7, 6001, 640, 523), (7, 6001, 384, 405), (8, 2051, 640, 4097),
             (8, 2051, 384, 4097), (9, 33, 640, 4097), (9, 33, 384, 3001), (9, 33, 1408, 4097)],
    (1, 0): [(0, 33, 4224, 2), (0, 33, 6272, 2), (1, 33, 2176, 2101), (1, 33, 5248, 2101), (2, 33, 2176, 3001),
             (2, 33, 5248, 3001), (3, 131, 1152, 2101), (3, 4101, 1920, 77), (4, 131, 2176, 2101), (4, 131, 5248, 2101),
             (5, 9001, 1152, 33), (5, 701, 1920, 1501), (6, 9001, 2176, 33), (6, 9001, 5248, 33), (7, 13001, 640, 131),
             (7, 13001, 384, 100), (7, 13001, 1408, 131), (8, 22003, 640, 301), (8, 22003, 384, 301), (8, 22003, 1408, 301),
             (9, 33, 1152, 1501), (9, 22003, 1920, 2)],
    (1, 8): [(0, 33, 4224, 2), (0, 33, 6272, 2), (1, 33, 2176, 2101), (1, 33, 5248, 2101), (2, 33, 2176, 3001),
             (2, 33, 5248, 3001), (3, 131, 1152, 2101), (3, 1001, 1920, 203), (4, 131, 2176, 2101), (4, 131, 5248, 2101),
             (5, 131, 1152, 4097), (5, 203, 1920, 4097), (6, 203, 2176, 2101), (6, 203, 5248, 2101), (7, 523, 640, 3001),
             (7, 523, 384, 3001), (7, 3001, 1408, 405), (8, 6001, 640, 701), (8, 6001, 384, 523), (8, 4101, 1408, 1501),
             (9, 33, 1152, 1501), (9, 3001, 1920, 11)],
}
# the other kinds, 8 experts: (shape, n, k, m); 4-bit codebooks have costs of their own
GROUPED_CASES = [(0, 33, 1152, 3), (1, 131, 640, 1501), (2, 77, 640, 3001), (3, 523, 896, 2101), (4, 3001, 384, 203),
                 (5, 2051, 640, 2101)]
CODEBOOK4_CASES = [(0, 33, 1152, 3), (1, 33, 640, 3001), (2, 77, 640, 2101), (3, 3001, 1152, 203), (4, 203, 384, 3001),
                   (5, 4101, 640, 701)]


def mx4_cases():
    """(MX4 rows, experts, shape, n, k, m)"""
    return [(a4, e, *c) for (a4, e), cs in MX4_CASES.items() for c in cs]


def grouped_cases():
    """(bits, kind, group, shape, n, k, m)"""
    return [(*f, *c) for f in FORMATS for c in (CODEBOOK4_CASES if f[:2] == (4, 1) else GROUPED_CASES)]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    subprocess.run([gxx, "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
                    os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host", "stages_model.cpp"), "-o", exe], check=True)

    def run(cases):
        text = "".join("%d %d %d %d %d %d %d\n" % c for c in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return run


def test_every_mx4_shape_runs_through_stages(plan):
    """Each shape has a product of three and more stages and one of an even number of them, with more scales
    a row than a load brings and not a multiple of them, whose last stage is not whole where a row can leave
    it so; those of at most two units a stage have one with few scales a row and a second stage too."""
    cases = mx4_cases()
    got = plan([(3, 4, a4, n, k, m, e) for a4, e, _, n, k, m in cases])
    assert [g[0] for g in got] == [c[2] for c in cases]
    for (a4, e), built in {(0, 0): 9, (0, 8): 10, (1, 0): 10, (1, 8): 10}.items():
        for shape in range(built):
            mine = [(k // 32, units, per) for (b, f, s, n, k, m), (_, units, per) in zip(cases, got) if (b, f, s) == (a4, e, shape)]
            per = mine[0][2]
            whole = per * (128 if a4 else 64) <= 128  # a row ends with a whole stage whatever its length
            long = [-(-units // per) for scales, units, _ in mine if scales > 16 and scales % 16 and (whole or units % per)]
            assert any(st >= 3 for st in long) and any(st % 2 == 0 for st in long), (a4, e, shape)
            if per <= 2:
                assert any(scales < 16 and units > per for scales, units, _ in mine), (a4, e, shape)
    # products of one matrix and two fp16 rows of 2048 and more do not reach the tiles
    assert not [c for c in cases if c[:2] == (0, 0) and c[5] <= 2 and c[4] >= 2048]


def test_every_grouped_shape_runs_through_stages(plan):
    cases = grouped_cases()
    got = plan([(kind, bits, 0, n, k, m, 8) for bits, kind, _, _, n, k, m in cases])
    assert [g[0] for g in got] == [c[3] for c in cases]
    for _, units, per in got:
        assert -(-units // per) >= 3 and (units % per or per == 1)
