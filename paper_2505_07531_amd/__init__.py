"""Python binding of libqx (include/qx.h): group-wise 3/4-bit quantized weights,
dequantized and multiplied by fp16 activations on an MI355X.

Argument marshalling only: every step of the path runs in the library's HIP
kernels. PyTorch supplies device memory and streams. If the library is not
built, ``load()`` builds it in-tree with hipcc; if it cannot be loaded, every
call raises -- there is no fallback.

Functions keep the C names:
  qx_pack_layout(desc, codes, scales=None, zeros=None, codebook=None) -> uint8 numpy blob
  qx_pack_q4x(desc, codes, scales, selectors, codebook) -> uint8 numpy blob
  qx_dequant(desc, packed, out_kind, out, stream=None)
  qx_gemv(desc, packed, x, y, stream=None)
  qx_gemv_a8(desc, packed, x, y, stream=None)
  qx_gemm(desc, packed, m, X, Y, stream=None)
  qx_quantize_a8(m, k, X, Xq, sx, stream=None)
  qx_gemm_a8(desc, packed, m, Xq, sx, Y, stream=None)
  qx_pack_mx4(desc, codes, scales) -> uint8 numpy blob
  qx_quantize_mx4(m, k, X, packed, stream=None)
  qx_gemm_a4(desc, packed, m, Xq, Y, stream=None)
  qx_gemm_grouped(desc, packed, m, X, offsets, Y, stream=None)
  qx_gemm_a4_grouped(desc, packed, m, Xq, offsets, Y, stream=None)
  qx_status_str(status)
Tensor arguments are torch CUDA tensors (HIP device memory); ``stream`` is a
torch stream (default: the current stream). Before a device call the binding
checks each tensor against the descriptor (device, dtype, contiguity, element
count) and raises ValueError without launching anything when one does not fit,
or does not lie on the current device, where the call launches.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import numpy as np

from . import _build

QX_UNIFORM, QX_CODEBOOK, QX_Q4X, QX_MX4 = 0, 1, 2, 3
QX_OUT_F16, QX_OUT_CODES = 0, 1
QX_OK, QX_E_ARG, QX_E_UNSUPPORTED, QX_E_SIZE, QX_E_HIP = 0, -1, -2, -3, -4

LIB_PATH = _build.LIB


class QxDesc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("k", ctypes.c_int32), ("bits", ctypes.c_int32),
                ("group", ctypes.c_int32), ("kind", ctypes.c_int32), ("flags", ctypes.c_uint32)]

    def __repr__(self):
        return (f"QxDesc(n={self.n}, k={self.k}, bits={self.bits}, group={self.group}, "
                f"kind={self.kind}, flags={self.flags})")


def desc(n: int, k: int, bits: int, group: int, kind: int, flags: int = 0) -> QxDesc:
    return QxDesc(n, k, bits, group, kind, flags)


class QxError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {qx_status_str(status)} ({status})")


_lib = None


def build() -> str:
    """Compile libqx.so for gfx950 in-tree (always recompiles)."""
    global _lib
    _lib = None
    return _build.build()


def load():
    """The loaded libqx (ctypes.CDLL); builds it first if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            _build.build()
        try:  # torch's HIP runtime first, so that libqx binds to the one that owns torch's memory
            import torch  # noqa: F401
        except ImportError:
            pass
        L = ctypes.CDLL(LIB_PATH)
        P, sz = ctypes.c_void_p, ctypes.c_size_t
        D = ctypes.POINTER(QxDesc)
        L.qx_pack_layout.argtypes = [D, P, P, P, P, P, sz, ctypes.POINTER(sz)]
        L.qx_pack_layout.restype = ctypes.c_int
        L.qx_pack_q4x.argtypes = [D, P, P, P, P, P, sz, ctypes.POINTER(sz)]
        L.qx_pack_q4x.restype = ctypes.c_int
        L.qx_dequant.argtypes = [D, P, ctypes.c_int, P, P]
        L.qx_dequant.restype = ctypes.c_int
        L.qx_gemv.argtypes = [D, P, P, P, P]
        L.qx_gemv.restype = ctypes.c_int
        L.qx_gemv_a8.argtypes = [D, P, P, P, P]
        L.qx_gemv_a8.restype = ctypes.c_int
        L.qx_gemm.argtypes = [D, P, ctypes.c_int32, P, P, P]
        L.qx_gemm.restype = ctypes.c_int
        L.qx_quantize_a8.argtypes = [ctypes.c_int32, ctypes.c_int32, P, P, P, P]
        L.qx_quantize_a8.restype = ctypes.c_int
        L.qx_gemm_a8.argtypes = [D, P, ctypes.c_int32, P, P, P, P]
        L.qx_gemm_a8.restype = ctypes.c_int
        i32 = ctypes.c_int32
        L.qx_pack_mx4.argtypes = [D, P, P, P, sz, ctypes.POINTER(sz)]
        L.qx_quantize_mx4.argtypes = [i32, i32, P, P, P]
        L.qx_gemm_a4.argtypes = [D, P, i32, P, P, P]
        L.qx_gemm_grouped.argtypes = [D, P, sz, i32, i32, P, P, P, P]
        L.qx_gemm_a4_grouped.argtypes = [D, P, sz, i32, i32, P, P, P, P]
        for f in (L.qx_pack_mx4, L.qx_quantize_mx4, L.qx_gemm_a4, L.qx_gemm_grouped, L.qx_gemm_a4_grouped):
            f.restype = ctypes.c_int
        L.qx_status_str.argtypes = [ctypes.c_int]
        L.qx_status_str.restype = ctypes.c_char_p
        _lib = L
    return _lib


def qx_status_str(status: int) -> str:
    return load().qx_status_str(int(status)).decode()


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def _check(st: int, where: str):
    if st != QX_OK:
        raise QxError(st, where)


def qx_packed_size(d: QxDesc) -> int:
    size = ctypes.c_size_t(0)
    _check(load().qx_pack_layout(ctypes.byref(d), None, None, None, None, None, 0,
                                 ctypes.byref(size)), "qx_pack_layout")
    return size.value


def qx_pack_layout(d: QxDesc, codes: np.ndarray, scales=None, zeros=None, codebook=None,
                   out: Optional[np.ndarray] = None) -> np.ndarray:
    """Packed blob (host uint8 array) of codes [n][k] and binary16 tables."""
    def c(a, dt):
        return None if a is None else np.ascontiguousarray(a, dtype=dt)
    codes, scales, zeros, codebook = c(codes, np.uint8), c(scales, np.uint16), c(zeros, np.uint16), \
        c(codebook, np.uint16)
    total = qx_packed_size(d)
    if out is None:
        out = np.empty(total, np.uint8)
    size = ctypes.c_size_t(0)
    _check(load().qx_pack_layout(ctypes.byref(d), _np_ptr(codes), _np_ptr(scales), _np_ptr(zeros),
                                 _np_ptr(codebook), _np_ptr(out), out.nbytes, ctypes.byref(size)),
           "qx_pack_layout")
    return out[:size.value]


def qx_pack_q4x(d: QxDesc, codes: np.ndarray, scales, selectors, codebook,
                out: Optional[np.ndarray] = None) -> np.ndarray:
    """Q4X blob (host uint8 array): codes [n][k], scales [n][k/64] (binary16 bits),
    selectors [n][k/64] (< 4), codebook [4][16] (binary16 bits)."""
    codes = np.ascontiguousarray(codes, dtype=np.uint8)
    scales = np.ascontiguousarray(scales, dtype=np.uint16)
    selectors = np.ascontiguousarray(selectors, dtype=np.uint8)
    codebook = np.ascontiguousarray(codebook, dtype=np.uint16)
    size = ctypes.c_size_t(0)
    L = load()
    _check(L.qx_pack_q4x(ctypes.byref(d), None, None, None, None, None, 0, ctypes.byref(size)),
           "qx_pack_q4x")
    if out is None:
        out = np.empty(size.value, np.uint8)
    _check(L.qx_pack_q4x(ctypes.byref(d), _np_ptr(codes), _np_ptr(scales), _np_ptr(selectors),
                         _np_ptr(codebook), _np_ptr(out), out.nbytes, ctypes.byref(size)), "qx_pack_q4x")
    return out[:size.value]


def qx_pack_mx4(d: QxDesc, codes: np.ndarray, scales, out: Optional[np.ndarray] = None) -> np.ndarray:
    """MX4 blob (host uint8 array): E2M1 codes [n][k] (< 16), E8M0 scales [n][k/32]."""
    codes = np.ascontiguousarray(codes, dtype=np.uint8)
    scales = np.ascontiguousarray(scales, dtype=np.uint8)
    size = ctypes.c_size_t(0)
    L = load()
    _check(L.qx_pack_mx4(ctypes.byref(d), None, None, None, 0, ctypes.byref(size)), "qx_pack_mx4")
    if codes.size != d.n * d.k or scales.size != d.n * d.k // 32:
        raise ValueError(f"codes {codes.shape} and scales {scales.shape} do not fit {d}")
    if out is None:
        out = np.empty(size.value, np.uint8)
    _check(L.qx_pack_mx4(ctypes.byref(d), _np_ptr(codes), _np_ptr(scales), _np_ptr(out), out.nbytes,
                         ctypes.byref(size)), "qx_pack_mx4")
    return out[:size.value]


def _chk(t, name: str, dtype, numel: int):
    """Check that `t` is a contiguous device tensor of `dtype` (None: any) holding at least
    `numel` elements (the kernels read and write exactly the sizes the descriptor implies)."""
    if t is None:
        raise ValueError(f"{name}: a device tensor is required")
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensors required")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if t.numel() < numel:
        raise ValueError(f"{name}: {t.numel()} elements, at least {numel} needed")


# The size follows from the six numbers alone, and asking the library for it took a good
# part of a small call (a 4096x4096 codebook-3 GEMV from Python 10.8 us with it, two stream
# objects' worth of torch.cuda.current_stream() and pointer objects; 7.2 us without).
@functools.lru_cache(maxsize=256)
def _blob_size(n: int, k: int, bits: int, group: int, kind: int, flags: int) -> int:
    size = ctypes.c_size_t(0)
    L = load()
    d = QxDesc(n, k, bits, group, kind, flags)
    if kind == QX_MX4:
        _check(L.qx_pack_mx4(ctypes.byref(d), None, None, None, 0, ctypes.byref(size)), "packed size")
        return size.value
    fn = L.qx_pack_q4x if kind == QX_Q4X else L.qx_pack_layout
    _check(fn(ctypes.byref(d), None, None, None, None, None, 0, ctypes.byref(size)), "packed size")
    return size.value


def qx_blob_size(d: QxDesc) -> int:
    """Bytes of the packed blob of `d` (any kind)."""
    return _blob_size(d.n, d.k, d.bits, d.group, d.kind, d.flags)


def _chk_packed(d: QxDesc, packed):
    import torch
    _chk(packed, "packed", torch.uint8, qx_blob_size(d))


def _rows(X, m: int, k: int, name: str):
    if X is not None and X.dim() == 2 and (X.shape[0] < m or X.shape[1] != k):
        raise ValueError(f"{name}: shape {tuple(X.shape)}, expected ({m}, {k})")


def _here(stream, *tensors):
    """The raw stream, once every tensor is known to lie on the current device (a launch goes to
    the current device, whatever the tensors' own)."""
    import torch
    at = torch._C._cuda_getDevice()
    for t in tensors:
        if t.get_device() != at:
            raise ValueError(f"tensor on {t.device}, but the current device is cuda:{at}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(at)  # no Stream object
    if stream.device.index != at:
        raise ValueError(f"stream of {stream.device}, but the current device is cuda:{at}")
    return stream.cuda_stream


def _new(stream, like, shape, dtype):
    """A new tensor for a call to write, on the device of `like`; for one on a given stream from that
    stream's own memory, since what the current stream freed it may still be writing."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    import torch
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def qx_dequant(d: QxDesc, packed, out_kind: int, out, stream=None) -> None:
    import torch
    _chk_packed(d, packed)
    _chk(out, "out", torch.float16 if out_kind == QX_OUT_F16 else torch.uint8, d.n * d.k)
    s = _here(stream, packed, out)
    _check(load().qx_dequant(ctypes.byref(d), packed.data_ptr(), out_kind, out.data_ptr(), s), "qx_dequant")


def qx_gemv(d: QxDesc, packed, x, y, stream=None) -> None:
    import torch
    _chk_packed(d, packed)
    _chk(x, "x", torch.float16, d.k)
    _chk(y, "y", torch.float16, d.n)
    s = _here(stream, packed, x, y)
    _check(load().qx_gemv(ctypes.byref(d), packed.data_ptr(), x.data_ptr(), y.data_ptr(), s), "qx_gemv")


def qx_gemv_a8(d: QxDesc, packed, x, y, stream=None) -> None:
    import torch
    _chk_packed(d, packed)
    _chk(x, "x", torch.float16, d.k)
    _chk(y, "y", torch.float16, d.n)
    s = _here(stream, packed, x, y)
    _check(load().qx_gemv_a8(ctypes.byref(d), packed.data_ptr(), x.data_ptr(), y.data_ptr(), s), "qx_gemv_a8")


def qx_gemm(d: QxDesc, packed, m: int, X, Y, stream=None) -> None:
    import torch
    m = int(m)
    _chk_packed(d, packed)
    _rows(X, m, d.k, "X")
    _chk(X, "X", torch.float16, m * d.k)
    _chk(Y, "Y", torch.float16, m * d.n)
    s = _here(stream, packed, X, Y)
    _check(load().qx_gemm(ctypes.byref(d), packed.data_ptr(), m, X.data_ptr(), Y.data_ptr(), s), "qx_gemm")


def qx_quantize_a8(m: int, k: int, X, Xq, sx, stream=None) -> None:
    import torch
    m, k = int(m), int(k)
    _chk(X, "X", torch.float16, m * k)
    _chk(Xq, "Xq", torch.int8, m * k)
    _chk(sx, "sx", torch.float32, m)
    s = _here(stream, X, Xq, sx)
    _check(load().qx_quantize_a8(m, k, X.data_ptr(), Xq.data_ptr(), sx.data_ptr(), s), "qx_quantize_a8")


def qx_gemm_a8(d: QxDesc, packed, m: int, Xq, sx, Y, stream=None) -> None:
    import torch
    m = int(m)
    _chk_packed(d, packed)
    _rows(Xq, m, d.k, "Xq")
    _chk(Xq, "Xq", torch.int8, m * d.k)
    _chk(sx, "sx", torch.float32, m)
    _chk(Y, "Y", torch.float16, m * d.n)
    s = _here(stream, packed, Xq, sx, Y)
    _check(load().qx_gemm_a8(ctypes.byref(d), packed.data_ptr(), m, Xq.data_ptr(), sx.data_ptr(), Y.data_ptr(), s),
           "qx_gemm_a8")


def qx_quantize_mx4(m: int, k: int, X, packed, stream=None) -> None:
    import torch
    m, k = int(m), int(k)
    _rows(X, m, k, "X")
    _chk(X, "X", torch.float16, m * k)
    _chk(packed, "packed", torch.uint8, m * k // 32 * 17)
    s = _here(stream, X, packed)
    _check(load().qx_quantize_mx4(m, k, X.data_ptr(), packed.data_ptr(), s), "qx_quantize_mx4")


def _mx4_rows(Xq, m: int, k: int):
    import torch
    _chk(Xq, "Xq", torch.uint8, m * k // 32 * 17)


def qx_gemm_a4(d: QxDesc, packed, m: int, Xq, Y, stream=None) -> None:
    import torch
    m = int(m)
    _chk_packed(d, packed)
    _mx4_rows(Xq, m, d.k)
    _chk(Y, "Y", torch.float16, m * d.n)
    s = _here(stream, packed, Xq, Y)
    _check(load().qx_gemm_a4(ctypes.byref(d), packed.data_ptr(), m, Xq.data_ptr(), Y.data_ptr(), s), "qx_gemm_a4")


def _chk_experts(d: QxDesc, packed, offsets):
    """(experts, bytes between their blobs) of a uint8 tensor [experts][at least the blob's size]."""
    import torch
    _chk(packed, "packed", torch.uint8, 0)
    if packed.dim() != 2 or packed.shape[1] % 16 or packed.shape[1] < qx_blob_size(d):
        raise ValueError(f"packed: shape {tuple(packed.shape)}, expected [experts][bytes], bytes a multiple of 16 "
                         f"and at least {qx_blob_size(d)}")
    _chk(offsets, "offsets", torch.int32, packed.shape[0] + 1)
    if offsets.numel() != packed.shape[0] + 1:
        raise ValueError(f"offsets: {offsets.numel()} elements, {packed.shape[0] + 1} expected")
    return packed.shape


def qx_gemm_grouped(d: QxDesc, packed, m: int, X, offsets, Y, stream=None) -> None:
    import torch
    m = int(m)
    experts, stride = _chk_experts(d, packed, offsets)
    _rows(X, m, d.k, "X")
    _chk(X, "X", torch.float16, m * d.k)
    _chk(Y, "Y", torch.float16, m * d.n)
    s = _here(stream, packed, X, offsets, Y)
    _check(load().qx_gemm_grouped(ctypes.byref(d), packed.data_ptr(), stride, experts, m, X.data_ptr(),
                                  offsets.data_ptr(), Y.data_ptr(), s), "qx_gemm_grouped")


def qx_gemm_a4_grouped(d: QxDesc, packed, m: int, Xq, offsets, Y, stream=None) -> None:
    import torch
    m = int(m)
    experts, stride = _chk_experts(d, packed, offsets)
    _mx4_rows(Xq, m, d.k)
    _chk(Y, "Y", torch.float16, m * d.n)
    s = _here(stream, packed, Xq, offsets, Y)
    _check(load().qx_gemm_a4_grouped(ctypes.byref(d), packed.data_ptr(), stride, experts, m, Xq.data_ptr(),
                                     offsets.data_ptr(), Y.data_ptr(), s), "qx_gemm_a4_grouped")


def quantize_mx4(X, stream=None) -> "PackedWeight":
    """An fp16 device tensor [m][k], weights or activations, rounded to MX4 where it lies."""
    import torch
    m, k = X.shape
    out = _new(stream, X, m * k // 32 * 17, torch.uint8)
    qx_quantize_mx4(m, k, X, out, stream)
    return PackedWeight._around(QxDesc(m, k, 4, 32, QX_MX4, 0), out, m * k // 32 * 17)


def quantize_a8(X, stream=None):
    """(Xq int8 [m][k], sx fp32 [m]) of an fp16 [m][k] device tensor."""
    import torch
    m, k = X.shape
    Xq = _new(stream, X, (m, k), torch.int8)
    sx = _new(stream, X, m, torch.float32)
    qx_quantize_a8(m, k, X, Xq, sx, stream)
    return Xq, sx


# ------------------------------------------------------------- conveniences
class PackedWeight:
    """A packed matrix resident in device memory, with its descriptor."""

    def __init__(self, d: QxDesc, blob: np.ndarray, device="cuda"):
        import torch
        self.desc = d
        self.nbytes = int(blob.size)
        self.data = torch.from_numpy(np.ascontiguousarray(blob)).to(device)

    @classmethod
    def from_quant(cls, q, device="cuda") -> "PackedWeight":
        """From an object with n, k, bits, group, kind, codes, scales, zeros, codebook
        (and selectors for Q4X; MX4: codes and E8M0 scales)."""
        d = desc(q.n, q.k, q.bits, q.group, q.kind)
        if q.kind == QX_MX4:
            return cls(d, qx_pack_mx4(d, q.codes, q.scales), device)
        if q.kind == QX_Q4X:
            return cls(d, qx_pack_q4x(d, q.codes, q.scales, q.selectors, q.codebook), device)
        return cls(d, qx_pack_layout(d, q.codes, q.scales, q.zeros, q.codebook), device)

    @classmethod
    def from_blob(cls, d: QxDesc, data) -> "PackedWeight":
        """Around a blob that is in device memory already (a uint8 tensor; not copied)."""
        _chk_packed(d, data)
        return cls._around(d, data, qx_blob_size(d))

    @classmethod
    def _around(cls, d: QxDesc, data, nbytes: int) -> "PackedWeight":
        self = cls.__new__(cls)
        self.desc, self.nbytes, self.data = d, nbytes, data
        return self

    def dequant(self, out_kind: int = QX_OUT_F16, stream=None):
        import torch
        dt = torch.float16 if out_kind == QX_OUT_F16 else torch.uint8
        out = _new(stream, self.data, (self.desc.n, self.desc.k), dt)
        qx_dequant(self.desc, self.data, out_kind, out, stream)
        return out

    def gemv(self, x, y=None, stream=None):
        import torch
        if y is None:
            y = _new(stream, x, self.desc.n, torch.float16)
        qx_gemv(self.desc, self.data, x, y, stream)
        return y

    def gemm_a8(self, Xq, sx, Y=None, stream=None):
        import torch
        m = Xq.shape[0]
        if Y is None:
            Y = _new(stream, Xq, (m, self.desc.n), torch.float16)
        qx_gemm_a8(self.desc, self.data, m, Xq, sx, Y, stream)
        return Y

    def gemv_a8(self, x, y=None, stream=None):
        import torch
        if y is None:
            y = _new(stream, x, self.desc.n, torch.float16)
        qx_gemv_a8(self.desc, self.data, x, y, stream)
        return y

    def gemm(self, X, Y=None, stream=None):
        import torch
        m = X.shape[0]
        if Y is None:
            Y = _new(stream, X, (m, self.desc.n), torch.float16)
        qx_gemm(self.desc, self.data, m, X, Y, stream)
        return Y

    def gemm_a4(self, Xq: "PackedWeight", Y=None, stream=None):
        """Of the rows that quantize_mx4 wrote."""
        import torch
        m = _rows_of(Xq, self.desc.k)
        if Y is None:
            Y = _new(stream, Xq.data, (m, self.desc.n), torch.float16)
        qx_gemm_a4(self.desc, self.data, m, Xq.data, Y, stream)
        return Y


def _rows_of(Xq: PackedWeight, k: int) -> int:
    if Xq.desc.kind != QX_MX4 or Xq.desc.k != k:
        raise ValueError(f"rows of {Xq.desc}, expected QX_MX4 rows of k = {k}")
    return Xq.desc.n


class PackedExperts:
    """Packed matrices of one descriptor, resident in device memory, for products of rows that are
    sorted by expert."""

    def __init__(self, d: QxDesc, data):
        """data: uint8 device tensor [experts][bytes], a blob at the head of every row; bytes a
        multiple of 16 (not copied)."""
        self.desc, self.data = d, data

    @classmethod
    def stack(cls, weights) -> "PackedExperts":
        """From PackedWeights of one descriptor, copied side by side."""
        import torch
        if not weights:
            raise ValueError("no experts")
        d, size = weights[0].desc, weights[0].nbytes
        if any(bytes(w.desc) != bytes(d) for w in weights):
            raise ValueError("experts of different descriptors")
        data = torch.zeros((len(weights), (size + 15) // 16 * 16), dtype=torch.uint8, device=weights[0].data.device)
        for e, w in enumerate(weights):
            data[e, :size] = w.data[:size]
        return cls(d, data)

    def gemm(self, X, offsets, Y=None, stream=None):
        """Rows offsets[e] .. offsets[e+1] - 1 of X times expert e; offsets int32 on the device."""
        import torch
        m = X.shape[0]
        if Y is None:
            Y = _new(stream, X, (m, self.desc.n), torch.float16)
        qx_gemm_grouped(self.desc, self.data, m, X, offsets, Y, stream)
        return Y

    def gemm_a4(self, Xq: PackedWeight, offsets, Y=None, stream=None):
        """The same with MX4 weights and the rows that quantize_mx4 wrote."""
        import torch
        m = _rows_of(Xq, self.desc.k)
        if Y is None:
            Y = _new(stream, Xq.data, (m, self.desc.n), torch.float16)
        qx_gemm_a4_grouped(self.desc, self.data, m, Xq.data, offsets, Y, stream)
        return Y
