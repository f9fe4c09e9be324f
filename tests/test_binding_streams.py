"""Devices and streams of the binding's calls, of every kind, without a GPU: tensors of another device are
refused before a launch, and the outputs of a call on a given stream are allocated on that stream."""
import contextlib
from types import SimpleNamespace

import numpy as np
import pytest

import paper_2505_07531_amd as qx

torch = pytest.importorskip("torch")

KINDS = [(3, qx.QX_UNIFORM, 64), (4, qx.QX_CODEBOOK, 128), (4, qx.QX_Q4X, 64), (4, qx.QX_MX4, 32)]
N, K, M = 64, 256, 4


class Tensor:
    """Stand-in for a device tensor of device 1; nothing reaches the library."""
    is_cuda, device = True, "cuda:1"
    made = None  # the Allocations of a test

    def __init__(self, dtype, *shape):
        self.dtype, self.shape = dtype, shape

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def is_contiguous(self):
        return True

    def get_device(self):
        return 1

    def new_empty(self, shape, dtype=None):
        return self.made.empty(shape, dtype)

    def data_ptr(self):
        raise AssertionError("a pointer was taken: the call would have launched")

    def __getitem__(self, at):
        return self


def calls():
    """(name, kind, what a user calls with tensors t and a stream s)"""
    f16, i8, u8, f32, i32 = torch.float16, torch.int8, torch.uint8, torch.float32, torch.int32
    x, X, Xq, sx = Tensor(f16, K), Tensor(f16, M, K), Tensor(i8, M, K), Tensor(f32, M)
    yield "quantize_a8", None, lambda s: qx.quantize_a8(X, stream=s)
    yield "quantize_mx4", None, lambda s: qx.quantize_mx4(X, stream=s)
    for bits, kind, group in KINDS:
        d = qx.desc(N, K, bits, group, kind)
        w = qx.PackedWeight.from_blob(d, Tensor(u8, qx.qx_blob_size(d)))
        stride = (qx.qx_blob_size(d) + 15) // 16 * 16
        experts, off = qx.PackedExperts(d, Tensor(u8, 2, stride)), Tensor(i32, 3)
        yield "dequant", kind, lambda s, w=w: w.dequant(stream=s)
        yield "codes", kind, lambda s, w=w: w.dequant(qx.QX_OUT_CODES, stream=s)
        yield "gemv", kind, lambda s, w=w: w.gemv(x, stream=s)
        yield "gemm", kind, lambda s, w=w: w.gemm(X, stream=s)
        yield "grouped", kind, lambda s, e=experts, off=off: e.gemm(X, off, stream=s)
        if kind == qx.QX_MX4:
            rows = qx.PackedWeight.from_blob(qx.desc(M, K, 4, 32, kind), Tensor(u8, M * K // 32 * 17))
            yield "gemm_a4", kind, lambda s, w=w, rows=rows: w.gemm_a4(rows, stream=s)
            yield "grouped_a4", kind, lambda s, e=experts, rows=rows, off=off: e.gemm_a4(rows, off, stream=s)
        else:
            yield "gemv_a8", kind, lambda s, w=w: w.gemv_a8(x, stream=s)
            yield "gemm_a8", kind, lambda s, w=w: w.gemm_a8(Xq, sx, stream=s)


CALLS = list(calls())
IDS = [f"{name}-{kind}" for name, kind, _ in CALLS]


class Allocations:
    """Stands in for torch's streams and allocator: on which stream each output was allocated."""

    def __init__(self, monkeypatch, current):
        self.now, self.on = None, []
        monkeypatch.setattr(torch, "empty", self.empty)
        monkeypatch.setattr(Tensor, "made", self)
        monkeypatch.setattr(torch.cuda, "stream", self.stream)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 5, raising=False)

    def empty(self, shape, dtype=None, device=None):
        self.on.append(self.now)
        return Tensor(dtype, *(shape if isinstance(shape, tuple) else (shape,)))

    @contextlib.contextmanager
    def stream(self, s):
        before, self.now = self.now, s
        yield
        self.now = before


@pytest.mark.parametrize("name,kind,call", CALLS, ids=IDS)
def test_tensors_of_another_device_are_refused(monkeypatch, name, kind, call):
    Allocations(monkeypatch, current=0)
    with pytest.raises(ValueError, match="current device"):
        call(None)


@pytest.mark.parametrize("name,kind,call", CALLS, ids=IDS)
def test_a_stream_of_another_device_is_refused(monkeypatch, name, kind, call):
    Allocations(monkeypatch, current=1)
    with pytest.raises(ValueError, match="current device"):
        call(SimpleNamespace(device=SimpleNamespace(index=0), cuda_stream=3))


@pytest.mark.parametrize("name,kind,call", CALLS, ids=IDS)
def test_outputs_are_allocated_on_the_stream_that_writes_them(monkeypatch, name, kind, call):
    """What the current stream freed it may still be writing."""
    made = Allocations(monkeypatch, current=1)
    given = SimpleNamespace(device=SimpleNamespace(index=1), cuda_stream=3)
    for stream in (given, None):
        made.on.clear()
        with pytest.raises(AssertionError, match="pointer"):  # all checks passed
            call(stream)
        assert made.on == [stream] * (2 if name == "quantize_a8" else 1)
