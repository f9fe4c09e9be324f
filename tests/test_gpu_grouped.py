"""Products grouped by expert on the GPU in the uniform, codebook and Q4X formats: every block shape, rows
of no expert, and a layer of experts, against the oracle in 64 bits (test_gpu_mx4.py runs these formats at
more offsets and sizes)."""
import numpy as np
import pytest

from oracle import mx4
from test_gpu_mx4 import activations, check_grouped, experts_of, random_mx4, run_grouped, to_dev
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


def test_layer_of_experts_from_fp16_weights(gpu):
    """Weights rounded to MX4 on the device and stacked, rows rounded to MX4, up and down products, on a
    stream of their own: as the oracle's steps, and bit for bit what the current stream gives."""
    import torch
    hid, ffn, m = 384, 256, 90
    rng = np.random.default_rng(12)
    ups = [rng.standard_normal((ffn, hid)).astype(np.float16) * np.float16(0.05) for _ in range(3)]
    downs = [rng.standard_normal((hid, ffn)).astype(np.float16) * np.float16(0.05) for _ in range(3)]
    x, off = activations(hid, 4, m), [0, 31, 31, 90]
    dx, doff = to_dev(x), to_dev(np.asarray(off, np.int32))

    def layer(stream):
        up = gpu.PackedExperts.stack([gpu.quantize_mx4(to_dev(w)) for w in ups])
        down = gpu.PackedExperts.stack([gpu.quantize_mx4(to_dev(w)) for w in downs])
        torch.cuda.synchronize()
        h = up.gemm_a4(gpu.quantize_mx4(dx, stream=stream), doff, stream=stream)
        y = down.gemm(h, doff, stream=stream)
        torch.cuda.synchronize()
        return h.cpu().numpy(), y.cpu().numpy()

    h, y = layer(None)
    h2, y2 = layer(torch.cuda.Stream())
    assert np.array_equal(h.view(np.uint16), h2.view(np.uint16)) and np.array_equal(y.view(np.uint16), y2.view(np.uint16))
    check_grouped(h, mx4.levels(*mx4.quantize(x)), [mx4.levels(*mx4.quantize(w)) for w in ups], off, 0)
    check_grouped(y, h, [mx4.dequant(*mx4.quantize(w)) for w in downs], off, 0)


@pytest.mark.parametrize("call", ["quantize", "dequant", "gemv", "gemm", "gemm_a4", "grouped", "grouped_a4"])
def test_outputs_of_another_stream_are_not_what_this_one_still_writes(gpu, call):
    """A tensor that the current stream has yet to fill is dropped just before a call on another stream
    allocates an output of its size: that output is written once, by the call."""
    import torch
    n, k, m = 512, 512, 64
    w = gpu.PackedWeight.from_quant(random_mx4(n, k, 5))
    experts = gpu.PackedExperts.stack([w, w])
    x, off = to_dev(activations(k, 6, m)), to_dev(np.array([0, 20, m], np.int32))
    xq = gpu.quantize_mx4(x)
    calls = {"quantize": lambda s: gpu.quantize_mx4(x, stream=s).data, "dequant": lambda s: w.dequant(stream=s),
             "gemv": lambda s: w.gemv(x[0], stream=s), "gemm": lambda s: w.gemm(x, stream=s),
             "gemm_a4": lambda s: w.gemm_a4(xq, stream=s), "grouped": lambda s: experts.gemm(x, off, stream=s),
             "grouped_a4": lambda s: experts.gemm_a4(xq, off, stream=s)}
    want = calls[call](None).clone()
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        torch.cuda._sleep(20_000_000)
        dropped = torch.empty_like(want).fill_(3)
        del dropped
        got = calls[call](other)
        other.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("bits,kind,group,a4", [(4, 3, 32, False), (4, 3, 32, True), (3, 0, 64, False), (4, 1, 32, False)])
def test_most_rows_and_experts(gpu, bits, kind, group, a4):
    """65536 rows of 1024 experts, most of the experts with rows, some with very many."""
    n, k, experts, m = 24, 128, 1024, 65536
    rng = np.random.default_rng(2)
    count = rng.integers(0, 3, experts) * rng.integers(0, 40, experts)
    count[[5, 700, 1023]] += [1000, 3000, 500]
    off = np.minimum(np.concatenate([[0], np.cumsum(count)]), m)
    pe, ws = experts_of(gpu, bits, kind, group, n, k, 4, 19)
    pe = gpu.PackedExperts(pe.desc, pe.data.repeat(experts // 4, 1))
    x = activations(k, 8, m)
    y = run_grouped(gpu, pe, x, off, a4=a4)
    check_grouped(y, mx4.levels(*mx4.quantize(x)) if a4 else x, ws * (experts // 4), off, 0x5A5A)


@pytest.mark.parametrize("kind,bits,group", [(3, 4, 32), (0, 3, 64)])
def test_no_rows(gpu, kind, bits, group):
    import torch
    pe, _ = experts_of(gpu, bits, kind, group, 40, 256, 2, 1)
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    none = torch.empty(0, 256, dtype=torch.float16, device="cuda")
    assert pe.gemm(none, off).shape == (0, 40)
    if kind == 3:
        q = gpu.quantize_mx4(none)
        assert q.dequant().shape == (0, 256)
        assert pe.gemm_a4(q, off).shape == (0, 40)
        one = gpu.PackedWeight.from_blob(pe.desc, pe.data[0])
        assert one.gemm(none).shape == (0, 40) and one.gemm_a4(q).shape == (0, 40)
