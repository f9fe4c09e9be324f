"""MX4 and the products grouped by expert on the GPU, through the binding, against the oracle in 64
bits: the quantiser and the expansion bit for bit; products within what fp32 sums and one rounding to
fp16 can be off; rows of no expert left as they were.

Tolerance of a product over k terms: the terms are exact, an fp32 sum of them in any order is off by
at most k * 2^-23 of the sum of their magnitudes (2^-24 a step where a step rounds, twice that where
it cuts off), and the store rounds to fp16 by 2^-11 of the value, or 2^-25 below its normal range.
"""
import numpy as np
import pytest

import oracle
from oracle import mx4
import qx_inputs as qi
from helpers import activations, random_quant, to_dev
from test_mx4_plan import shape_cases

pytestmark = pytest.mark.gpu

FORMATS = [(b, kind, g) for b in (3, 4) for kind in (0, 1) for g in (32, 64, 128)] + [(4, 2, 64), (4, 3, 32)]


def check(y, x, w):
    """y against x @ w.T, all rows."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    ref, size = x @ w.T, np.abs(x) @ np.abs(w).T
    tol = x.shape[1] * 2.0**-23 * size
    tol = tol + 2.0**-11 * (np.abs(ref) + tol) + 2.0**-25
    off = np.abs(np.asarray(y, np.float64) - ref)
    assert np.all(off <= tol), (off / tol).max()  # false for NaN


def random_mx4(n, k, seed, lo=116, hi=124):
    rng = np.random.default_rng(seed)
    return qi.QuantWeight(n, k, 4, 32, 3, rng.integers(0, 16, (n, k), dtype=np.uint8),
                          scales=rng.integers(lo, hi, (n, k // 32), dtype=np.uint8))


def blob_of(codes, scales):
    return to_dev(mx4.pack(codes, scales))


def rows_of(qx, codes, scales):
    return qx.PackedWeight.from_blob(qx.desc(*codes.shape, 4, 32, qx.QX_MX4), blob_of(codes, scales))


# ------------------------------------------------------------------ quantise and expand
def quantise_inputs():
    rng = np.random.default_rng(7)
    every = np.arange(65536, dtype=np.uint16)  # every fp16 value beside others of its size
    yield "every", np.concatenate([every.reshape(-1, 128), rng.permutation(every).reshape(-1, 128)]).view(np.float16)
    grid = np.repeat(mx4.value(np.arange(16)), 8)[None]  # values, and the ties between them
    ties = np.tile(np.array([4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, 6.9, 5.004, 4.996, -0.25, -0.75, -1.25, -5]), 8)[None]
    x = np.concatenate([np.concatenate([grid, ties]) * 2.0**p for p in range(-24, 13)])
    yield "ties", x.astype(np.float16)
    w = np.zeros((9, 128), np.float16)
    w[1] = -0.0
    w[2, 5], w[3, 40], w[4, 100] = np.inf, np.nan, -np.inf
    w[5] = np.float16(6e-8)
    w[6] = 65504
    w[7, ::3] = 1e-7
    w[8] = rng.standard_normal(128)
    yield "wild", w
    for m, k in ((1, 128), (3, 1152), (257, 384), (5, 11008), (33, 4096)):
        yield f"{m}x{k}", (rng.standard_normal((m, k)) * 10.0 ** rng.integers(-5, 4, (m, 1))).astype(np.float16)


@pytest.mark.parametrize("name,x", list(quantise_inputs()), ids=lambda v: v if isinstance(v, str) else "")
def test_quantize_bit_exact(gpu, name, x):
    codes, scales = mx4.quantize(x)
    got = gpu.quantize_mx4(to_dev(x))
    c, s = mx4.unpack(got.data.cpu().numpy(), *x.shape)
    assert np.array_equal(s, scales)
    tame = np.repeat(scales != 255, 32, axis=-1)
    assert np.array_equal(c[tame], codes[tame])
    back = got.dequant().cpu().numpy()
    want = mx4.dequant(codes, scales)
    assert np.isnan(back[~tame]).all() and np.array_equal(back[tame].view(np.uint16), want[tame].view(np.uint16))
    assert np.array_equal(got.dequant(gpu.QX_OUT_CODES).cpu().numpy()[tame], codes[tame])


def test_dequant_every_code_and_scale(gpu):
    codes = np.tile(np.arange(16, dtype=np.uint8), (256, 8))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 4, -1)
    got = rows_of(gpu, codes, scales).dequant().cpu().numpy()
    want = mx4.dequant(codes, scales)
    assert np.isnan(got[255]).all()
    assert np.array_equal(got[:255].view(np.uint16), want[:255].view(np.uint16))


@pytest.mark.parametrize("m,k", [(1, 128), (31, 2176)])
def test_quantize_writes_its_blob_alone(gpu, m, k):
    import torch
    x = to_dev(activations(k, 5, m))
    size = m * k // 32 * 17
    buf = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    gpu.qx_quantize_mx4(m, k, x, buf[:size])
    assert (buf[size:] == 0xA5).all()
    assert np.array_equal(buf[:size].cpu().numpy(), mx4.pack(*mx4.quantize(x.cpu().numpy())))


# ------------------------------------------------------------------ products
SHAPES = [(1, 128), (3, 384), (37, 256), (64, 1152), (130, 4096), (5, 11008), (1001, 640), (4097, 512), (272, 8192)]


@pytest.mark.parametrize("n,k", SHAPES)
@pytest.mark.parametrize("m", [1, 2, 5, 16, 17, 33, 64, 77])
def test_gemm(gpu, n, k, m):
    q = random_mx4(n, k, n + k)
    x = activations(k, n + m, m)
    pw = gpu.PackedWeight.from_quant(q)
    w = mx4.dequant(q.codes, q.scales)
    check(pw.gemm(to_dev(x)).cpu().numpy(), x, w)
    if m == 1:
        check(pw.gemv(to_dev(x[0])).cpu().numpy()[None], x, w)


@pytest.mark.parametrize("n,k", SHAPES)
@pytest.mark.parametrize("m", [1, 2, 5, 16, 17, 33, 64, 77])
def test_gemm_a4(gpu, n, k, m):
    q = random_mx4(n, k, n + k)
    x = activations(k, n + m, m)
    codes, scales = mx4.quantize(x)
    got = gpu.PackedWeight.from_quant(q).gemm_a4(gpu.quantize_mx4(to_dev(x))).cpu().numpy()
    check(got, mx4.levels(codes, scales), mx4.levels(q.codes, q.scales))


@pytest.mark.parametrize("n,k,m", [(300, 1408, 129), (515, 384, 700), (256, 1024, 2049), (2050, 896, 513)])
def test_many_rows(gpu, n, k, m):
    q = random_mx4(n, k, n + k)
    x = activations(k, n + m, m)
    pw = gpu.PackedWeight.from_quant(q)
    check(pw.gemm(to_dev(x)).cpu().numpy(), x, mx4.dequant(q.codes, q.scales))
    codes, scales = mx4.quantize(x)
    check(pw.gemm_a4(gpu.quantize_mx4(to_dev(x))).cpu().numpy(), mx4.levels(codes, scales), mx4.levels(q.codes, q.scales))


@pytest.mark.parametrize("m", [1, 3, 16, 40, 130, 600])
def test_one_hot_rows_give_columns(gpu, m):
    """Every code and every scale of the fp16 range: a column of W', exactly."""
    n, k = 200, 1152
    q = random_mx4(n, k, 3, lo=104, hi=140)
    w = mx4.dequant(q.codes, q.scales)
    at = np.random.default_rng(m).integers(0, k, m)
    x = np.zeros((m, k), np.float16)
    x[np.arange(m), at] = 1
    pw = gpu.PackedWeight.from_quant(q)
    assert np.array_equal(pw.gemm(to_dev(x)).cpu().numpy(), w[:, at].T)
    if m == 1:
        assert np.array_equal(pw.gemv(to_dev(x[0])).cpu().numpy(), w[:, at[0]])
    assert np.array_equal(pw.gemm_a4(gpu.quantize_mx4(to_dev(x))).cpu().numpy(), w[:, at].T)


@pytest.mark.parametrize("m", [1, 8, 60, 300])
def test_nan_and_extreme_scales(gpu, m):
    """A NaN block makes NaN of its row's products and of no others; scales far outside of fp16 cancel
    where both sides are MX4."""
    n, k = 70, 512
    q = random_mx4(n, k, 11)
    q.scales[33, 5] = 255
    x = activations(k, 21, m)
    pw = gpu.PackedWeight.from_quant(q)
    w = mx4.levels(q.codes, q.scales)
    got = pw.gemm(to_dev(x)).cpu().numpy()
    rest = np.arange(n) != 33
    assert np.isnan(got[:, 33]).all()
    check(got[:, rest], x, w[rest])
    codes, scales = mx4.quantize(x)
    wild = scales.copy()
    wild[m - 1, 2] = 255
    got = pw.gemm_a4(rows_of(gpu, codes, wild)).cpu().numpy()
    assert np.isnan(got[m - 1]).all() and np.isnan(got[:, 33]).all()
    check(got[:m - 1, rest], mx4.levels(codes, scales)[:m - 1], w[rest])
    far = gpu.PackedWeight.from_quant(qi.QuantWeight(n, k, 4, 32, 3, q.codes, scales=np.full_like(q.scales, 190)))
    got = far.gemm_a4(rows_of(gpu, codes, np.full_like(scales, 57))).cpu().numpy()
    check(got, mx4.value(codes) * 2.0**-35, mx4.value(q.codes) * 2.0**28)


def test_inf_and_nan_activations_stay_in_their_rows(gpu):
    n, k, m = 48, 256, 40
    q = random_mx4(n, k, 2)
    q.codes[:] |= 1  # no weight is zero
    x = activations(k, 4, m)
    x[3, 7], x[20, 100] = np.inf, np.nan
    got = gpu.PackedWeight.from_quant(q).gemm(to_dev(x)).cpu().numpy()
    rest = np.setdiff1d(np.arange(m), [3, 20])
    assert np.isnan(got[20]).all() and np.isinf(got[3]).all()
    check(got[rest], x[rest], mx4.dequant(q.codes, q.scales))


# ------------------------------------------------------------------ grouped by expert
def experts_of(qx, bits, kind, group, n, k, experts, seed):
    """PackedExperts, and their W' in fp64."""
    if kind == 3:
        qs = [random_mx4(n, k, seed + e) for e in range(experts)]
        ws = [mx4.dequant(q.codes, q.scales) for q in qs]
    elif kind == 2:
        from test_gpu_q4x import _ref, random_q4x
        qs = [random_q4x(n, k, seed + e) for e in range(experts)]
        ws = [_ref(q) for q in qs]
    else:
        qs = [random_quant(n, k, bits, group, kind, seed + e) for e in range(experts)]
        ws = [oracle.dequant(q.codes, group, kind, q.scales, q.zeros, q.codebook) for q in qs]
    return qx.PackedExperts.stack([qx.PackedWeight.from_quant(q) for q in qs]), ws


def check_grouped(y, x, ws, offsets, fill):
    covered = np.zeros(len(x), bool)
    for e, w in enumerate(ws):
        a, b = offsets[e], offsets[e + 1]
        covered[a:b] = True
        if b > a:
            check(y[a:b], x[a:b], w)
    assert (y[~covered].view(np.uint16) == fill).all()


def run_grouped(qx, pe, x, offsets, a4=False, fill=0x5A5A):
    import torch
    m, n = len(x), pe.desc.n
    buf = torch.full((m * n + 64,), fill, dtype=torch.int16, device="cuda").view(torch.float16)
    y = buf[:m * n].view(m, n)
    off = to_dev(np.asarray(offsets, np.int32))
    if a4:
        pe.gemm_a4(qx.quantize_mx4(to_dev(x)), off, Y=y)
    else:
        pe.gemm(to_dev(x), off, Y=y)
    assert (buf[m * n:].view(torch.int16) == fill).all()  # nothing past the last row
    return y.cpu().numpy()


OFFSETS = {
    "even": [0, 8, 16, 24, 32], "one": [0, 0, 1, 1, 1], "none": [5, 5, 5, 5, 5], "first": [0, 70, 70, 70, 70],
    "last": [0, 0, 0, 0, 33], "gaps": [3, 3, 20, 90, 95], "ragged": [0, 1, 18, 147, 300], "many": [2, 260, 261, 700, 905],
}


@pytest.mark.parametrize("name", OFFSETS)
@pytest.mark.parametrize("bits,kind,group", FORMATS)
def test_grouped(gpu, bits, kind, group, name):
    n, k, off = 83, 384, OFFSETS[name]
    m = off[-1] + (7 if name in ("gaps", "none", "many") else 0)
    pe, ws = experts_of(gpu, bits, kind, group, n, k, 4, 17)
    x = activations(k, 31, m)
    check_grouped(run_grouped(gpu, pe, x, off), x, ws, off, 0x5A5A)


@pytest.mark.parametrize("name", OFFSETS)
def test_grouped_a4(gpu, name):
    n, k, off = 83, 384, OFFSETS[name]
    m = off[-1] + (7 if name in ("gaps", "none", "many") else 0)
    pe, ws = experts_of(gpu, 4, 3, 32, n, k, 4, 17)
    x = activations(k, 31, m)
    check_grouped(run_grouped(gpu, pe, x, off, a4=True), mx4.levels(*mx4.quantize(x)), ws, off, 0x5A5A)


@pytest.mark.parametrize("bits,kind,group", [(4, 3, 32), (4, 0, 128), (3, 1, 64)])
@pytest.mark.parametrize("experts", [1, 63, 64, 65, 130, 300])
def test_grouped_number_of_experts(gpu, bits, kind, group, experts):
    rng = np.random.default_rng(experts)
    count = rng.integers(0, 4, experts) * rng.integers(0, 2, experts)
    count[-1] = 2
    off = np.concatenate([[0], np.cumsum(count)])
    pe, ws = experts_of(gpu, bits, kind, group, 33, 128, experts, 5)
    x = activations(128, 8, off[-1])
    check_grouped(run_grouped(gpu, pe, x, off), x, ws, off, 0x5A5A)
    if kind == 3:
        check_grouped(run_grouped(gpu, pe, x, off, a4=True), mx4.levels(*mx4.quantize(x)), ws, off, 0x5A5A)


@pytest.mark.parametrize("bits,kind,group", [(4, 3, 32), (3, 0, 64)])
@pytest.mark.parametrize("n,k,sizes", [(1, 128, [1, 0, 3]), (257, 4096, [40, 2, 0, 5]), (1376, 1408, [0, 200, 17]),
                                       (512, 896, [513, 300]), (100, 11008, [1, 1, 1, 1, 1, 1])])
def test_grouped_sizes(gpu, bits, kind, group, n, k, sizes):
    off = np.concatenate([[0], np.cumsum(sizes)])
    pe, ws = experts_of(gpu, bits, kind, group, n, k, len(sizes), 9)
    x = activations(k, 12, off[-1])
    check_grouped(run_grouped(gpu, pe, x, off), x, ws, off, 0x5A5A)
    if kind == 3:
        check_grouped(run_grouped(gpu, pe, x, off, a4=True), mx4.levels(*mx4.quantize(x)), ws, off, 0x5A5A)


@pytest.mark.parametrize("a4", [False, True])
@pytest.mark.parametrize("off", [[-5, 3, 2**31 - 1, 40, 40], [30, 20, 10, 0, -2**31], [0, 50, 0, 50, 50]])
def test_grouped_offsets_out_of_range_stay_in_bounds(gpu, a4, off):
    """Offsets are held to the rows that there are; nothing is written outside of Y (run_grouped)."""
    pe, ws = experts_of(gpu, 4, 3, 32, 83, 384, 4, 17)
    x = activations(384, 31, 50)
    y = run_grouped(gpu, pe, x, off, a4=a4)
    if off[0] == -5:  # rows 0..2, 3..49, none (50 to 40), none
        check_grouped(y, mx4.levels(*mx4.quantize(x)) if a4 else x, ws, [0, 3, 50, 50, 50], 0x5A5A)
    if off[0] == 30:
        assert (y.view(np.uint16) == 0x5A5A).all()


def test_grouped_one_expert_is_gemm(gpu):
    pe, ws = experts_of(gpu, 4, 3, 32, 130, 640, 1, 2)
    x = activations(640, 6, 50)
    check(run_grouped(gpu, pe, x, [0, 50]), x, ws[0])


@pytest.mark.parametrize("a4,shape,n,k,m,experts", shape_cases())
def test_every_block_shape(gpu, a4, shape, n, k, m, experts):
    """Every shape of the tiles, alone or grouped (test_mx4_plan shows which product takes which)."""
    if experts:
        rng = np.random.default_rng(n + m)
        off = np.concatenate([[0], np.sort(rng.integers(0, m + 1, experts - 1)), [m]])
        pe, ws = experts_of(gpu, 4, 3, 32, n, k, experts, 7)
        x = activations(k, 3, m)
        check_grouped(run_grouped(gpu, pe, x, off, a4=bool(a4)), mx4.levels(*mx4.quantize(x)) if a4 else x, ws, off, 0x5A5A)
        return
    q = random_mx4(n, k, 7)
    x = activations(k, 3, m)
    pw = gpu.PackedWeight.from_quant(q)
    if a4:
        check(pw.gemm_a4(gpu.quantize_mx4(to_dev(x))).cpu().numpy(), mx4.levels(*mx4.quantize(x)), mx4.levels(q.codes, q.scales))
    else:
        check(pw.gemm(to_dev(x)).cpu().numpy(), x, mx4.dequant(q.codes, q.scales))


@pytest.mark.parametrize("a4", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_grouped_random_offsets(gpu, a4, seed):
    """Many experts of one small matrix each, any number of rows of any of them."""
    rng = np.random.default_rng(seed)
    experts, n, k = int(rng.integers(1, 1025)), 19, 128
    count = rng.integers(0, 40, experts) * (rng.random(experts) < rng.choice([0.05, 0.5, 1.0]))
    off = np.concatenate([[0], np.cumsum(count)]) + rng.integers(0, 5)
    m = int(off[-1]) + int(rng.integers(0, 5))
    q = random_mx4(n * experts, k, seed)
    size = mx4.packed_size(n, k)
    blobs = np.stack([mx4.pack(q.codes[e * n:(e + 1) * n], q.scales[e * n:(e + 1) * n]) for e in range(experts)])
    data = np.zeros((experts, (size + 15) // 16 * 16), np.uint8)
    data[:, :size] = blobs
    pe = gpu.PackedExperts(gpu.desc(n, k, 4, 32, gpu.QX_MX4), to_dev(data))
    ws = mx4.dequant(q.codes, q.scales).reshape(experts, n, k)
    x = activations(k, seed, m)
    check_grouped(run_grouped(gpu, pe, x, off, a4=a4), mx4.levels(*mx4.quantize(x)) if a4 else x, ws, off, 0x5A5A)


# ------------------------------------------------------------------ as they are used
def test_expert_layer_captured_and_replayed(gpu):
    """Up and down products of a layer of experts, the rows between them rounded to MX4, captured once
    and replayed with other rows and another split of them; every replay equals the eager calls."""
    import torch
    hid, ffn, experts, m = 512, 384, 6, 40
    up, wu = experts_of(gpu, 4, 3, 32, ffn, hid, experts, 3)
    down, wd = experts_of(gpu, 4, 3, 32, hid, ffn, experts, 40)
    x = torch.empty(m, hid, dtype=torch.float16, device="cuda")
    off = torch.empty(experts + 1, dtype=torch.int32, device="cuda")

    def layer():
        h = up.gemm(x, off)
        return h, down.gemm(torch.relu(h), off), down.gemm_a4(gpu.quantize_mx4(torch.relu(h)), off)

    def fill(seed):
        rng = np.random.default_rng(seed)
        xs = activations(hid, seed, m)
        cut = np.concatenate([[0], np.sort(rng.integers(0, m + 1, experts - 1)), [m]])
        x.copy_(to_dev(xs))
        off.copy_(to_dev(cut.astype(np.int32)))
        return xs, cut

    fill(0)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        layer()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = layer()
    for seed in range(1, 5):
        xs, cut = fill(seed)
        g.replay()
        torch.cuda.synchronize()
        eager = layer()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)
        h, y, y4 = (t.cpu().numpy() for t in out)
        check_grouped(h, xs, wu, cut, 0)
        r = np.maximum(h, 0)
        check_grouped(y, r, wd, cut, 0)
        check_grouped(y4, mx4.levels(*mx4.quantize(r)), wd, cut, 0)


def test_other_stream_and_repeats(gpu):
    """A call on a stream of its own, given as an argument; the same bits every time."""
    import torch
    n, k, m = 1001, 1408, 300
    q = random_mx4(n, k, 8)
    pw = gpu.PackedWeight.from_quant(q)
    x = to_dev(activations(k, 9, m))
    pe, _ = experts_of(gpu, 4, 3, 32, 257, k, 3, 4)
    off = to_dev(np.array([0, 100, 117, 300], np.int32))
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), []
    for _ in range(3):
        with torch.cuda.stream(side):  # allocations belong to the stream that uses them
            xq = gpu.quantize_mx4(x, stream=side)
            got.append([pw.gemm(x, stream=side), pw.gemm(x[:7].clone(), stream=side), pw.gemv(x[0], stream=side),
                        pw.gemm_a4(xq, stream=side), pe.gemm(x, off, stream=side), pe.gemm_a4(xq, off, stream=side)])
    side.synchronize()
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
    check(got[0][0].cpu().numpy(), x.cpu().numpy(), mx4.dequant(q.codes, q.scales))


def test_rows_of_y_at_any_even_address(gpu):
    import torch
    n, k, m = 45, 256, 21
    q = random_mx4(n, k, 8)
    x = activations(k, 9, m)
    pw = gpu.PackedWeight.from_quant(q)
    for at in (1, 3):
        buf = torch.full((m * n + 8,), 7.0, dtype=torch.float16, device="cuda")
        pw.gemm(to_dev(x), Y=buf[at:at + m * n].view(m, n))
        check(buf[at:at + m * n].view(m, n).cpu().numpy(), x, mx4.dequant(q.codes, q.scales))
        assert (buf[:at] == 7).all() and (buf[at + m * n:] == 7).all()


def test_codes_past_four_gigabytes(gpu):
    """Experts whose blobs lie more than 2^32 bytes apart, and a matrix of more than 2^32 elements."""
    import torch
    n, k = 16, 256
    q = random_mx4(n, k, 1)
    size = gpu.qx_blob_size(gpu.desc(n, k, 4, 32, gpu.QX_MX4))
    data = torch.empty((3, (1 << 31) + 4096), dtype=torch.uint8, device="cuda")
    for e in range(3):
        data[e, :size] = blob_of((q.codes + e) % 16, q.scales)
    pe = gpu.PackedExperts(gpu.desc(n, k, 4, 32, gpu.QX_MX4), data)
    x = activations(k, 2, 9)
    off = [0, 2, 5, 9]
    ws = [mx4.dequant((q.codes + e) % 16, q.scales) for e in range(3)]
    check_grouped(run_grouped(gpu, pe, x, off), x, ws, off, 0x5A5A)
    check_grouped(run_grouped(gpu, pe, x, off, a4=True), mx4.levels(*mx4.quantize(x)), ws, off, 0x5A5A)
    del data, pe
    n, k = (1 << 17) + 3, 1 << 15  # 2.1 GB of codes, 4.3e9 elements
    base = torch.randint(0, 256, (1 << 20,), dtype=torch.uint8, device="cuda")
    blob = torch.full((n * k // 32 * 17,), 120, dtype=torch.uint8, device="cuda")
    blob[:n * k // 2].view(-1, k // 2)[:] = base[:k // 2]
    blob[(n - 1) * k // 2:n * k // 2] = base[k // 2:k]
    pw = gpu.PackedWeight.from_blob(gpu.desc(n, k, 4, 32, gpu.QX_MX4), blob)
    x = activations(k, 3, 2)
    c = np.stack([base[i * k // 2:(i + 1) * k // 2].cpu().numpy() for i in range(2)])
    w = mx4.value(np.stack([c & 15, c >> 4], -1).reshape(2, k)) * 2.0**-7
    for m in (1, 2):
        y = pw.gemm(to_dev(x[:m])).cpu().numpy()
        check(y[:, [0, n - 2, n - 1]], x[:m], w[[0, 0, 1]])
    y = pw.gemm_a4(gpu.quantize_mx4(to_dev(x))).cpu().numpy()
    check(y[:, [0, n - 2, n - 1]], mx4.levels(*mx4.quantize(x)), w[[0, 0, 1]])


@pytest.mark.parametrize("m", [1, 2])
@pytest.mark.parametrize("n,k", [(77, 2048), (1, 2176), (31, 4096), (4099, 4224), (33, 8320), (65, 16384), (9, 32768)])
def test_one_and_two_rows(gpu, n, k, m):
    """Long rows of weights, whole and in part of a wave's turn; a row of X that is NaN stays alone."""
    q = random_mx4(n, k, n + k)
    x = activations(k, 9, m)
    pw = gpu.PackedWeight.from_quant(q)
    w = mx4.dequant(q.codes, q.scales)
    y = pw.gemm(to_dev(x)).cpu().numpy()
    check(y, x, w)
    x2 = np.concatenate([x[:1], np.full((1, k), np.nan, np.float16)])[:m]
    again = pw.gemm(to_dev(x2)).cpu().numpy()
    assert np.array_equal(again[:1].view(np.uint16), y[:1].view(np.uint16)) and np.isnan(again[1:]).all()
