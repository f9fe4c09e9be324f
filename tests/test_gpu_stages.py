"""Every block shape of the MX4 and the grouped products through several stages (test_stage_cases.py shows which
product takes which), and rows of any length, bit for bit.

Inputs are such that no sum rounds: weights and rows are multiples of small powers of two, and the sum of the
terms' magnitudes is less than 2^24 times the least step of a term, so that every partial sum in any order is
a value of fp32. The outputs are then the exact sums rounded once to fp16: a block of k that is lost, taken
twice or with another's scale shows, whatever the length of the row."""
import numpy as np
import pytest

import oracle
from oracle import mx4, q4x
import qx_inputs as qi
from helpers import to_dev
from test_gpu_mx4 import blob_of, rows_of, run_grouped
from test_grouped_plan import FORMATS
from test_stage_cases import grouped_cases, mx4_cases

pytestmark = pytest.mark.gpu


def exact(x, w):
    """x @ w.T rounded once, for inputs whose sums do not round (checked)."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    steps = [2.0 ** np.floor(np.log2(np.abs(a[a != 0]).min())) for a in (x, w)]
    for a, s in zip((x, w), steps):
        assert (a / s == np.round(a / s)).all()
    assert x.shape[1] * np.abs(x).max() * np.abs(w).max() < 2.0**24 * steps[0] * steps[1]
    with np.errstate(over="ignore"):
        return (x @ w.T).astype(np.float16)


def same(y, want):
    y = np.asarray(y)
    bad = np.argwhere(y != want)
    assert bad.size == 0, (len(bad), bad[:4].tolist(), y[y != want][:4], want[y != want][:4])  # NaN is never equal


def mx4_weights(n, k, seed, lo=127, hi=128):
    """Codes and scales of steps of 0.5 and 1 (lo = hi: of one)."""
    rng = np.random.default_rng(seed)
    return rng.integers(0, 16, (n, k), dtype=np.uint8), rng.integers(lo, hi + 1, (n, k // 32), dtype=np.uint8)


def packed(qx, codes, scales):
    return qx.PackedWeight.from_blob(qx.desc(*codes.shape, 4, 32, qx.QX_MX4), blob_of(codes, scales))


def fp16_rows(m, k, seed, top=3):
    return np.random.default_rng(seed).integers(-top, top + 1, (m, k)).astype(np.float16)


def split_of(m, experts, seed):
    """Uneven rows of the experts, rows of no expert at both ends where there are enough."""
    low, high = (1, m - 2) if m > 9 else (0, m)
    cut = np.sort(np.random.default_rng(seed).integers(low, high + 1, experts - 1))
    return np.concatenate([[low], cut, [high]])


def same_grouped(y, x, ws, off, fill=0x5A5A):
    covered = np.zeros(len(x), bool)
    for e, w in enumerate(ws):
        a, b = off[e], off[e + 1]
        covered[a:b] = True
        if b > a:
            same(y[a:b], exact(x[a:b], w))
    assert (y[~covered].view(np.uint16) == fill).all()


@pytest.mark.parametrize("a4,experts,shape,n,k,m", mx4_cases())
def test_mx4_shapes(gpu, a4, experts, shape, n, k, m):
    cs = [mx4_weights(n, k, 10 + e) for e in range(max(experts, 1))]
    ws = [mx4.levels(*c) for c in cs]
    if a4:
        codes, scales = mx4_weights(m, k, 3, 126, 127)
        x, rows = mx4.levels(codes, scales), rows_of(gpu, codes, scales)
    else:
        x = fp16_rows(m, k, 3)
    if not experts:
        w = packed(gpu, *cs[0])
        same((w.gemm_a4(rows) if a4 else w.gemm(to_dev(x))).cpu().numpy(), exact(x, ws[0]))
        return
    pe, off = gpu.PackedExperts.stack([packed(gpu, *c) for c in cs]), split_of(m, experts, n + m)
    if not a4:
        same_grouped(run_grouped(gpu, pe, x, off), x, ws, off)
        return
    import torch
    y = torch.full((m, n), 0x5A5A, dtype=torch.int16, device="cuda").view(torch.float16)
    pe.gemm_a4(rows, to_dev(off.astype(np.int32)), Y=y)
    same_grouped(y.cpu().numpy(), x, ws, off)


def small_weights(qx, bits, kind, group, n, k, seed):
    """(PackedWeight, W') of a format, with levels that are multiples of 0.5 up to 16."""
    rng = np.random.default_rng(seed)
    codes, G = rng.integers(0, 2**bits, (n, k), dtype=np.uint8), k // group
    if kind == 2:
        q = qi.QuantWeight(n, k, 4, 64, 2, codes, scales=rng.choice([0.5, 1.0], (n, G)).astype(np.float16).view(np.uint16),
                           codebook=rng.integers(-8, 9, (4, 16)).astype(np.float16).view(np.uint16),
                           selectors=rng.integers(0, 4, (n, G), dtype=np.uint8))
        return qx.PackedWeight.from_quant(q), q4x.dequant(q.codes, q.scales, q.selectors, q.codebook)
    if kind == 1:
        book = (rng.integers(-16, 17, (n, G, 2**bits)) / 2).astype(np.float16)
        q = qi.QuantWeight(n, k, bits, group, 1, codes, codebook=book.view(np.uint16))
    else:
        q = qi.QuantWeight(n, k, bits, group, 0, codes, scales=rng.choice([0.5, 1.0], (n, G)).astype(np.float16).view(np.uint16),
                           zeros=rng.integers(0, 2**bits, (n, G)).astype(np.float16).view(np.uint16))
    return qx.PackedWeight.from_quant(q), oracle.dequant(q.codes, group, kind, q.scales, q.zeros, q.codebook)


@pytest.mark.parametrize("bits,kind,group,shape,n,k,m", grouped_cases())
def test_grouped_shapes(gpu, bits, kind, group, shape, n, k, m):
    both = [small_weights(gpu, bits, kind, group, n, k, 20 + e) for e in range(8)]
    pe, ws = gpu.PackedExperts.stack([w for w, _ in both]), [w for _, w in both]
    x, off = fp16_rows(m, k, 4), split_of(m, 8, n + m)
    same_grouped(run_grouped(gpu, pe, x, off), x, ws, off)


# ------------------------------------------------------------------ long rows
LONG = [(31, 4224), (77, 8320), (19, 11008), (65, 16384), (9, 32768)]


@pytest.mark.parametrize("n,k", LONG)
@pytest.mark.parametrize("m", [1, 2, 3, 9, 40, 200])
def test_mx4_long_rows(gpu, n, k, m):
    codes, scales = mx4_weights(n, k, n)
    w, x = mx4.levels(codes, scales), fp16_rows(m, k, m)
    pw = packed(gpu, codes, scales)
    same(pw.gemm(to_dev(x)).cpu().numpy(), exact(x, w))
    if m == 1:
        same(pw.gemv(to_dev(x[0])).cpu().numpy(), exact(x, w)[0])
    xc, xs = mx4_weights(m, k, m, 127, 127)
    same(pw.gemm_a4(rows_of(gpu, xc, xs)).cpu().numpy(), exact(mx4.levels(xc, xs), w))


@pytest.mark.parametrize("n,k", [(31, 4224), (19, 11008), (9, 32768)])
@pytest.mark.parametrize("m", [1, 2, 3, 9, 40, 200])
def test_mx4_one_block_of_a_long_row(gpu, n, k, m):
    """Rows of X that are zero but for one block, the first and last of them and some between: nothing of
    that block is lost among other terms, and W' of any scale of fp16's range."""
    rng = np.random.default_rng(m)
    codes, scales = mx4_weights(n, k, n, 112, 130)
    pw = packed(gpu, codes, scales)
    w = mx4.dequant(codes, scales)
    at = np.concatenate([[k // 32 - 1, 0, k // 32 - 2], rng.integers(0, k // 32, m)])[:m] * 32 + rng.integers(0, 32, m)
    x = np.zeros((m, k), np.float16)
    x[np.arange(m), at] = rng.choice([-1.0, 1.0, 2.0], m)
    want = (w[:, at].T * x[np.arange(m), at][:, None]).astype(np.float16)
    same(pw.gemm(to_dev(x)).cpu().numpy(), want)
    same(pw.gemm_a4(gpu.quantize_mx4(to_dev(x))).cpu().numpy(), want)
    if m == 1:
        same(pw.gemv(to_dev(x[0])).cpu().numpy(), want[0])


@pytest.mark.parametrize("bits,kind,group", FORMATS)
@pytest.mark.parametrize("n,k,m", [(19, 11008, 5), (33, 16384, 40)])
def test_grouped_long_rows(gpu, bits, kind, group, n, k, m):
    both = [small_weights(gpu, bits, kind, group, n, k, 40 + e) for e in range(3)]
    pe, ws = gpu.PackedExperts.stack([w for w, _ in both]), [w for _, w in both]
    x, off = fp16_rows(m, k, 4, 2), split_of(m, 3, 1)
    same_grouped(run_grouped(gpu, pe, x, off), x, ws, off)


@pytest.mark.parametrize("a4", [False, True])
@pytest.mark.parametrize("n,k,m", [(19, 11008, 5), (33, 16384, 40), (65, 8320, 300)])
def test_mx4_grouped_long_rows(gpu, a4, n, k, m):
    cs = [mx4_weights(n, k, 50 + e) for e in range(3)]
    pe, ws, off = gpu.PackedExperts.stack([packed(gpu, *c) for c in cs]), [mx4.levels(*c) for c in cs], split_of(m, 3, 1)
    x = fp16_rows(m, k, 6, 2)  # 0, 1 and 2: the same in MX4
    x[:, ::32] = 2             # a block's scale is that of its largest
    same_grouped(run_grouped(gpu, pe, x, off, a4=a4), x, ws, off)
