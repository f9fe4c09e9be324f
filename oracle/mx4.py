"""Oracle of the MX4 format and of products grouped by expert (test infrastructure).

MX4 is the microscaled 4-bit floating point of the OCP Microscaling specification (v1.0, MXFP4):
blocks of 32 consecutive elements of a row with E2M1 codes (sign, two exponent bits of bias 1, one
fraction bit) and one E8M0 scale byte e, worth 2^(e - 127), 255 for NaN.

  W'[n,k] = fp16_RNE( value(q[n,k]) * 2^(e[n,j] - 127) ),   j = k // 32

Quantization of a block: e - 127 = floor(log2 max|x|) - 2, x * 2^(127 - e) to the nearest value, ties
to the even code, magnitudes above 6 to 6; zeros give e = 0, a block with an infinity or NaN e = 255.

Blob: the codes row by row, two a byte, the even one in the low bits, then the scale bytes row by row.
"""
from __future__ import annotations

import numpy as np

GROUP = 32


def value(q) -> np.ndarray:
    """E2M1 codes as fp64, by the definition of the fields."""
    q = np.asarray(q, np.int64)
    sign, e, f = q >> 3, (q >> 1) & 3, q & 1
    mag = np.where(e == 0, f * 0.5, (1 + f / 2) * 2.0 ** (e - 1.0))
    return np.where(sign == 1, -mag, mag)


def scale(e) -> np.ndarray:
    e = np.asarray(e, np.int64)
    return np.where(e == 255, np.nan, np.ldexp(1.0, e - 127))


def levels(codes, scales) -> np.ndarray:
    """value * scale of codes [n][k] in fp64, not rounded."""
    return value(codes) * np.repeat(scale(scales), GROUP, axis=-1)


def dequant(codes, scales) -> np.ndarray:
    """fp16 W' [n][k]."""
    with np.errstate(over="ignore", invalid="ignore"):
        return levels(codes, scales).astype(np.float16)


def quantize(x16):
    """(codes uint8 [m][k], scales uint8 [m][k/32]) of fp16 rows."""
    x = np.asarray(x16, np.float16).astype(np.float64)
    m, k = x.shape
    b = x.reshape(m, k // GROUP, GROUP)
    top = np.abs(b).max(-1)
    wild = ~np.isfinite(b).all(-1)
    e = np.where((top > 0) & ~wild, np.frexp(np.where(wild, 1.0, top))[1] - 1 - 2 + 127, 0)
    grid = value(np.arange(8))
    with np.errstate(invalid="ignore"):
        a = np.minimum(np.ldexp(np.abs(b), (127 - e)[..., None]), 6.0)
    a = np.where(wild[..., None], 0.0, a)
    dist = np.abs(a[..., None] - grid)
    best = dist.min(-1, keepdims=True)
    near = dist == best  # one, or two neighbours in a tie: of those the even code
    code = np.where(near.sum(-1) == 1, near.argmax(-1),
                    np.where(near.argmax(-1) % 2 == 0, near.argmax(-1), near.argmax(-1) + 1))
    code = code + 8 * np.signbit(b)
    return code.astype(np.uint8).reshape(m, k), np.where(wild, 255, e).astype(np.uint8)


def packed_size(n: int, k: int) -> int:
    return n * k // 2 + n * k // GROUP


def pack(codes, scales) -> np.ndarray:
    codes = np.asarray(codes, np.uint8)
    return np.concatenate([(codes[:, 0::2] | codes[:, 1::2] << 4).reshape(-1), np.asarray(scales, np.uint8).reshape(-1)])


def unpack(blob, n: int, k: int):
    """(codes [n][k], scales [n][k/32])"""
    blob = np.asarray(blob, np.uint8)
    by = blob[:n * k // 2].reshape(n, k // 2)
    codes = np.empty((n, k), np.uint8)
    codes[:, 0::2], codes[:, 1::2] = by & 15, by >> 4
    return codes, blob[n * k // 2:packed_size(n, k)].reshape(n, k // GROUP)


def grouped(x, ws, offsets) -> np.ndarray:
    """Rows offsets[e] .. offsets[e+1] - 1 of x times ws[e] transposed, in fp64; NaN in rows of no expert."""
    x = np.asarray(x, np.float64)
    y = np.full((x.shape[0], ws[0].shape[0]), np.nan)
    for e, w in enumerate(ws):
        y[offsets[e]:offsets[e + 1]] = x[offsets[e]:offsets[e + 1]] @ np.asarray(w, np.float64).T
    return y
