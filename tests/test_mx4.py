"""MX4 without a GPU: the oracle's pins, the host packer against it, the refusals of every entry
point and the checks of the binding (nothing is launched here)."""
import ctypes

import numpy as np
import pytest

import paper_2505_07531_amd as qx
from oracle import mx4

P = ctypes.c_void_p


def _desc(n=4, k=128, bits=4, group=32, kind=None):
    return qx.desc(n, k, bits, group, qx.QX_MX4 if kind is None else kind)


# ------------------------------------------------------------------ oracle
def test_values_of_all_codes():
    want = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert mx4.value(np.arange(16)).tolist() == want + [-v for v in want]
    assert np.signbit(mx4.value([8]))[0]


def test_quantize_a_block_by_hand():
    x = np.zeros((1, 128), np.float16)
    # max 7 -> e = 0 (scale 1): ties 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4; 7 -> 6
    x[0, :12] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5.01, -0.25, 6.9, -0.0]
    x[0, 32:34] = [3, -1]     # max 3: scale 2^(1-2), 6 and -2
    x[0, 64] = np.inf         # no scale
    codes, scales = mx4.quantize(x)
    assert scales.tolist() == [[127, 126, 255, 0]]
    assert codes[0, :12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 15, 8, 7, 8]
    assert codes[0, 32:34].tolist() == [7, 12]
    assert np.isnan(mx4.dequant(codes, scales)[0, 64:96]).all()
    assert (mx4.dequant(codes, scales)[0, 96:] == 0).all()


def test_quantize_is_nearest_and_its_blobs_are_exact_in_fp16():
    rng = np.random.default_rng(0)
    bits = rng.integers(0, 0x7C00, (64, 512)) | rng.integers(0, 2, (64, 512)) << 15
    x = bits.astype(np.uint16).view(np.float16)
    x[32:] = (rng.standard_normal((32, 512)) * 10.0 ** rng.integers(-8, 4, (32, 1))).astype(np.float16)
    codes, scales = mx4.quantize(x)
    lv = mx4.levels(codes, scales)
    assert np.array_equal(lv, mx4.dequant(codes, scales).astype(np.float64))
    # no level of the block is nearer (those above 6 are held to it: nearest anyway)
    every = mx4.value(np.arange(16)) * np.repeat(mx4.scale(scales), 32, -1)[..., None]
    assert (np.abs(lv - x) <= np.abs(every - x.astype(np.float64)[..., None]).min(-1)).all()
    top = np.abs(x.astype(np.float64)).reshape(64, -1, 32).max(-1)
    s = mx4.scale(scales)
    assert ((top >= 4 * s) & (top < 8 * s) | (top == 0)).all()


def test_pack_and_unpack():
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 16, (5, 384), dtype=np.uint8)
    scales = rng.integers(0, 256, (5, 12), dtype=np.uint8)
    blob = mx4.pack(codes, scales)
    assert blob.size == mx4.packed_size(5, 384) == 5 * 384 * 17 // 32
    c, s = mx4.unpack(blob, 5, 384)
    assert np.array_equal(c, codes) and np.array_equal(s, scales)
    assert blob[0] == codes[0, 0] | codes[0, 1] << 4 and blob[192] == codes[1, 0] | codes[1, 1] << 4


# ------------------------------------------------------------------ host packer
@pytest.mark.parametrize("n,k", [(1, 128), (3, 1152), (5, 11008), (0, 256)])
def test_pack_mx4_matches_oracle_bytes(n, k):
    rng = np.random.default_rng(n + k)
    codes = rng.integers(0, 16, (n, k), dtype=np.uint8)
    scales = rng.integers(0, 256, (n, k // 32), dtype=np.uint8)
    d = _desc(n, k)
    assert qx.qx_blob_size(d) == mx4.packed_size(n, k)
    assert np.array_equal(qx.qx_pack_mx4(d, codes, scales), mx4.pack(codes, scales))


def _st(fn):
    try:
        fn()
    except qx.QxError as e:
        return e.status
    return qx.QX_OK


def test_pack_mx4_errors():
    codes, scales = np.zeros((2, 128), np.uint8), np.zeros((2, 4), np.uint8)
    assert _st(lambda: qx.qx_pack_mx4(_desc(2), codes, scales)) == qx.QX_OK
    assert _st(lambda: qx.qx_pack_mx4(_desc(2), codes + 16, scales)) == qx.QX_E_ARG
    assert _st(lambda: qx.qx_pack_mx4(_desc(2, group=64), codes, scales)) == qx.QX_E_ARG
    assert _st(lambda: qx.qx_pack_mx4(_desc(2, bits=3), codes, scales)) == qx.QX_E_ARG
    assert _st(lambda: qx.qx_pack_mx4(_desc(2, kind=qx.QX_CODEBOOK), codes, scales)) == qx.QX_E_ARG
    assert _st(lambda: qx.qx_pack_mx4(_desc(2), codes, scales, out=np.empty(135, np.uint8))) == qx.QX_E_SIZE
    with pytest.raises(ValueError):
        qx.qx_pack_mx4(_desc(2), codes[:1], scales)
    assert _st(lambda: qx.qx_pack_layout(_desc(2), codes)) == qx.QX_E_ARG  # the other packers refuse the kind
    assert _st(lambda: qx.qx_pack_q4x(_desc(2), codes, codes, codes, codes)) == qx.QX_E_ARG


# ------------------------------------------------------------------ refusals before a launch
def test_mx4_calls_refuse_before_launch():
    lib, d = qx.load(), _desc()
    r = ctypes.byref(d)
    assert lib.qx_gemv(r, P(16), None, P(16), None) == qx.QX_E_ARG
    assert lib.qx_gemm(r, P(8), 3, P(16), P(16), None) == qx.QX_E_ARG
    assert lib.qx_dequant(r, P(16), 5, P(16), None) == qx.QX_E_ARG
    assert lib.qx_gemv(ctypes.byref(_desc(group=64)), P(16), P(16), P(16), None) == qx.QX_E_ARG
    # int8 activations are not built for the kind
    assert lib.qx_gemv_a8(r, P(16), P(16), P(16), None) == qx.QX_E_UNSUPPORTED
    assert lib.qx_gemm_a8(r, P(16), 2, P(16), P(16), P(16), None) == qx.QX_E_UNSUPPORTED
    q = lib.qx_quantize_mx4
    assert q(-1, 128, P(16), P(16), None) == qx.QX_E_ARG
    assert q(1, 96, P(16), P(16), None) == qx.QX_E_ARG
    assert q(1, 0, P(16), P(16), None) == qx.QX_E_ARG
    assert q(1, (1 << 20) + 128, P(16), P(16), None) == qx.QX_E_ARG
    assert q(1, 128, None, P(16), None) == qx.QX_E_ARG
    assert q(1, 128, P(16), P(24), None) == qx.QX_E_ARG
    assert q(0, 128, None, None, None) == qx.QX_OK
    a4 = lib.qx_gemm_a4
    assert a4(None, P(16), 1, P(16), P(16), None) == qx.QX_E_ARG
    assert a4(ctypes.byref(qx.desc(4, 128, 4, 32, qx.QX_UNIFORM)), P(16), 1, P(16), P(16), None) == qx.QX_E_UNSUPPORTED
    assert a4(r, P(16), -1, P(16), P(16), None) == qx.QX_E_ARG
    assert a4(r, P(16), 65537, P(16), P(16), None) == qx.QX_E_ARG
    assert a4(r, P(16), 1, P(8), P(16), None) == qx.QX_E_ARG
    assert a4(r, P(16), 1, P(16), P(17), None) == qx.QX_E_ARG
    assert a4(r, P(16), 1, P(16), None, None) == qx.QX_E_ARG
    assert a4(r, None, 0, None, None, None) == qx.QX_OK


@pytest.mark.parametrize("call", ["qx_gemm_grouped", "qx_gemm_a4_grouped"])
def test_grouped_calls_refuse_before_launch(call):
    fn = getattr(qx.load(), call)
    d = _desc()
    size = qx.qx_blob_size(d)  # 272, a multiple of 16
    ok = dict(d=ctypes.byref(d), packed=P(16), stride=size, experts=3, m=4, X=P(16), offsets=P(16), Y=P(16))

    def st(**kw):
        a = {**ok, **kw}
        return fn(a["d"], a["packed"], a["stride"], a["experts"], a["m"], a["X"], a["offsets"], a["Y"], None)

    for bad in (dict(d=None), dict(packed=None), dict(packed=P(24)), dict(stride=size - 16), dict(stride=size + 8),
                dict(experts=-1), dict(experts=1025), dict(m=-1), dict(m=65537), dict(X=None), dict(X=P(8)),
                dict(offsets=None), dict(offsets=P(18)), dict(Y=None), dict(Y=P(17)),
                dict(d=ctypes.byref(qx.desc(4, 128, 4, 64, qx.QX_MX4)))):
        assert st(**bad) == qx.QX_E_ARG, bad
    for nothing in (dict(m=0), dict(experts=0), dict(d=ctypes.byref(_desc(n=0)))):
        assert st(**nothing, packed=None, X=None, offsets=None, Y=None) == qx.QX_OK
    if call == "qx_gemm_a4_grouped":
        assert st(d=ctypes.byref(qx.desc(4, 128, 4, 32, qx.QX_UNIFORM)), stride=4096) == qx.QX_E_UNSUPPORTED
    else:
        assert st(d=ctypes.byref(qx.desc(4, 128, 2, 32, qx.QX_UNIFORM)), stride=4096) == qx.QX_E_UNSUPPORTED


class _Fake:
    """Stand-in for a device tensor: the binding's checks run, nothing launches."""

    def __init__(self, dtype, *shape, contiguous=True, cuda=True):
        self.dtype, self.shape, self._c, self.is_cuda = dtype, shape, contiguous, cuda

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def is_contiguous(self):
        return self._c

    def get_device(self):
        raise AssertionError("past the checks: the call would have launched")

    def data_ptr(self):
        raise AssertionError("a pointer was taken: the call would have launched")


def test_binding_checks_tensors():
    torch = pytest.importorskip("torch")
    u8, f16, i32 = torch.uint8, torch.float16, torch.int32
    d = _desc(64, 256)
    size = qx.qx_blob_size(d)
    blob, X, Y, Xq = _Fake(u8, size), _Fake(f16, 4, 256), _Fake(f16, 4, 64), _Fake(u8, 4 * 136)
    for bad in ((_Fake(u8, 4 * 136 - 1), Y), (_Fake(f16, 4 * 136), Y), (_Fake(u8, 4 * 136, contiguous=False), Y),
                (Xq, _Fake(f16, 4 * 64 - 1)), (Xq, _Fake(torch.float32, 4, 64)), (Xq, _Fake(f16, 4, 64, cuda=False))):
        with pytest.raises(ValueError):
            qx.qx_gemm_a4(d, blob, 4, *bad)
    with pytest.raises(ValueError):
        qx.qx_gemm_a4(d, _Fake(u8, size - 1), 4, Xq, Y)
    for bad in ((_Fake(f16, 4, 255), blob), (_Fake(torch.bfloat16, 4, 256), blob), (X, _Fake(u8, 4 * 136 - 1))):
        with pytest.raises(ValueError):
            qx.qx_quantize_mx4(4, 256, *bad)
    experts, off = _Fake(u8, 3, size), _Fake(i32, 4)
    for e, o in ((_Fake(u8, 3 * size), off), (_Fake(u8, 3, size - 16), off), (_Fake(u8, 3, size + 8), off),
                 (experts, _Fake(i32, 3)), (experts, _Fake(i32, 5)), (experts, _Fake(torch.int64, 4)),
                 (experts, _Fake(i32, 4, cuda=False)), (experts, None)):
        with pytest.raises(ValueError):
            qx.qx_gemm_grouped(d, e, 4, X, o, Y)
        with pytest.raises(ValueError):
            qx.qx_gemm_a4_grouped(d, e, 4, Xq, o, Y)
    with pytest.raises(ValueError):
        qx.qx_gemm_grouped(d, experts, 4, _Fake(f16, 3, 256), off, Y)
    w = qx.PackedWeight.from_blob(d, blob)
    with pytest.raises(ValueError):  # rows of another length, or not MX4
        w.gemm_a4(qx.PackedWeight.from_blob(_desc(4, 128), _Fake(u8, 4 * 68)))
    with pytest.raises(ValueError):
        w.gemm_a4(qx.PackedWeight.from_blob(qx.desc(4, 256, 4, 32, qx.QX_UNIFORM), _Fake(u8, 4096)))


def test_tensors_of_another_device_are_refused(monkeypatch):
    """A launch goes to the current device: tensors, or a stream, of another one are an error."""
    from types import SimpleNamespace as NS
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 5, raising=False)
    here, there = (NS(get_device=lambda i=i: i, device=NS(index=i), cuda_stream=7 + i) for i in (0, 1))
    with pytest.raises(ValueError):
        qx._here(None, here, there)
    with pytest.raises(ValueError):
        qx._here(there, here, here)
    assert qx._here(here, here, here) == 7
    assert qx._here(None, here) == 5


def test_products_of_more_tiles_than_a_launch_takes_are_refused():
    """Before anything is enqueued: the sizes alone decide."""
    lib = qx.load()
    big = ctypes.byref(_desc(2**31 - 1, 128))
    assert lib.qx_gemv(big, P(16), P(16), P(16), None) == qx.QX_E_UNSUPPORTED
    assert lib.qx_gemm(big, P(16), 1, P(16), P(16), None) == qx.QX_E_UNSUPPORTED
    for m in (2, 65536):
        assert lib.qx_gemm(big, P(16), m, P(16), P(16), None) == qx.QX_E_UNSUPPORTED
        assert lib.qx_gemm_a4(big, P(16), m, P(16), P(16), None) == qx.QX_E_UNSUPPORTED
    for d in (_desc(2**31 - 1, 128), qx.desc(2**31 - 1, 128, 3, 64, qx.QX_CODEBOOK), qx.desc(2**31 - 1, 128, 4, 128, qx.QX_UNIFORM),
              qx.desc(2**31 - 1, 128, 4, 64, qx.QX_Q4X)):
        stride = qx.qx_blob_size(d) // 16 * 16 + 16
        for m in (1, 300, 65536):
            assert lib.qx_gemm_grouped(ctypes.byref(d), P(16), stride, 1024, m, P(16), P(16), P(16), None) == qx.QX_E_UNSUPPORTED
    stride = qx.qx_blob_size(_desc(2**31 - 1, 128)) // 16 * 16 + 16
    assert lib.qx_gemm_a4_grouped(big, P(16), stride, 1024, 65536, P(16), P(16), P(16), None) == qx.QX_E_UNSUPPORTED


def test_mx4_calls_of_another_device_are_refused(monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)

    class There(_Fake):
        device = "cuda:1"

        def get_device(self):
            return 1

    d = _desc(64, 256)
    blob, x, X, Y = There(torch.uint8, qx.qx_blob_size(d)), There(torch.float16, 256), There(torch.float16, 4, 256), There(torch.float16, 64 * 256)
    with pytest.raises(ValueError, match="current device"):
        qx.qx_dequant(d, blob, qx.QX_OUT_F16, Y)
    with pytest.raises(ValueError, match="current device"):
        qx.qx_gemv(d, blob, x, Y)
    with pytest.raises(ValueError, match="current device"):
        qx.qx_gemm(d, blob, 4, X, Y)


def test_a_stack_of_no_experts_or_of_different_ones_is_refused():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        qx.PackedExperts.stack([])
    a, b = _desc(64, 256), _desc(32, 256)
    with pytest.raises(ValueError):
        qx.PackedExperts.stack([qx.PackedWeight.from_blob(d, _Fake(torch.uint8, qx.qx_blob_size(d))) for d in (a, b)])
