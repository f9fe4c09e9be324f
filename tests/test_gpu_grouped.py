"""Products grouped by expert on the GPU in the uniform, codebook and Q4X formats: every block shape, rows
of no expert, and a layer of experts, against the oracle in 64 bits (test_gpu_mx4.py runs these formats at
more offsets and sizes)."""
import numpy as np
import pytest

from test_gpu_mx4 import activations, check_grouped, experts_of, run_grouped, to_dev
from test_grouped_plan import FORMATS, SHAPE_CASES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", range(len(SHAPE_CASES)))
@pytest.mark.parametrize("bits,kind,group", FORMATS)
def test_every_block_shape(gpu, bits, kind, group, shape):
    """Every shape in every format, the experts' rows uneven (test_grouped_plan shows which product takes
    which), with rows of no expert at both ends where there are enough."""
    n, k, m, experts = SHAPE_CASES[shape]
    rng = np.random.default_rng(n + m)
    low, high = (2, m - 3) if m > 9 else (0, m)
    off = np.concatenate([[low], np.sort(rng.integers(low, high + 1, experts - 1)), [high]])
    pe, ws = experts_of(gpu, bits, kind, group, n, k, experts, 7)
    x = activations(k, 3, m)
    check_grouped(run_grouped(gpu, pe, x, off), x, ws, off, 0x5A5A)


@pytest.mark.parametrize("bits,kind,group", FORMATS)
def test_one_hot_rows_give_columns(gpu, bits, kind, group):
    """Row r of X is 1 at column c(r): the product is that column of W', bit for bit."""
    n, k, m = 70, 640, 640
    pe, ws = experts_of(gpu, bits, kind, group, n, k, 2, 23)
    cols = np.random.default_rng(1).permutation(k)
    x = np.zeros((m, k), np.float16)
    x[np.arange(m), cols] = 1
    for off in ([0, 640, 640], [0, 9, 17], [0, 40, 80], [0, 320, 640]):
        y = run_grouped(gpu, pe, x, off)
        for e in (0, 1):
            a, b = off[e], off[e + 1]
            assert np.array_equal(y[a:b].astype(np.float64), ws[e][:, cols[a:b]].T)


@pytest.mark.parametrize("bits,kind,group", [(3, 1, 64), (4, 0, 128), (4, 2, 64)])
@pytest.mark.parametrize("m", [3, 40, 200, 900])
def test_inf_and_nan_stay_in_their_rows(gpu, bits, kind, group, m):
    """Infinities and NaN in some rows of an expert leave its other rows and the other expert finite."""
    n, k = 600, 512
    pe, ws = experts_of(gpu, bits, kind, group, n, k, 2, 11)
    x = activations(k, 5, m)
    cut = m // 3
    bad = [0, cut, m - 1]
    x[bad, [1, 300, 511]] = [np.inf, np.nan, -np.inf]
    y = run_grouped(gpu, pe, x, [0, cut, m])
    good = np.setdiff1d(np.arange(m), bad)
    assert not np.isfinite(y[bad]).all(axis=1).any()
    clean = x.copy()
    clean[bad] = 0
    again = run_grouped(gpu, pe, clean, [0, cut, m])
    assert np.array_equal(y[good].view(np.uint16), again[good].view(np.uint16))


def test_captured_with_new_offsets(gpu):
    """One captured product replayed with other offsets and rows: the shape follows m alone, and every
    replay is the eager product."""
    import torch
    n, k, m, experts = 300, 768, 130, 5
    pe, ws = experts_of(gpu, 3, 0, 64, n, k, experts, 3)
    x = torch.zeros(m, k, dtype=torch.float16, device="cuda")
    off = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    y = torch.zeros(m, n, dtype=torch.float16, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        pe.gemm(x, off, Y=y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        pe.gemm(x, off, Y=y)
    rng = np.random.default_rng(8)
    for it in range(4):
        xs = activations(k, 60 + it, m)
        o = np.concatenate([[0], np.sort(rng.integers(0, m + 1, experts - 1)), [m]]).astype(np.int32)
        x.copy_(to_dev(xs)), off.copy_(to_dev(o)), y.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        eager = run_grouped(gpu, pe, xs, o)
        assert np.array_equal(y.cpu().numpy().view(np.uint16), eager.view(np.uint16))
        check_grouped(y.cpu().numpy(), xs, ws, o, 0x5A5A)


def test_same_expert_bytes_twice(gpu):
    """The same bytes given twice are two experts."""
    import torch
    pe, ws = experts_of(gpu, 4, 0, 64, 90, 256, 1, 31)
    blob = pe.data[:1]
    two = gpu.PackedExperts(pe.desc, torch.cat([blob, blob]))
    x = activations(256, 9, 30)
    check_grouped(run_grouped(gpu, two, x, [0, 11, 30]), x, [ws[0], ws[0]], [0, 11, 30], 0x5A5A)
