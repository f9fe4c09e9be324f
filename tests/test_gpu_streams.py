"""Outputs of calls on a given stream, in the formats with int8 rows and without: test_gpu_grouped.py has the
same for MX4."""
import numpy as np
import pytest

from helpers import activations, random_quant, to_dev

pytestmark = pytest.mark.gpu

KINDS = [(3, 0, 64), (4, 1, 128), (4, 2, 64)]


def weight_of(qx, bits, kind, group, n, k):
    if kind == 2:
        from test_gpu_q4x import random_q4x
        return qx.PackedWeight.from_quant(random_q4x(n, k, 5))
    return qx.PackedWeight.from_quant(random_quant(n, k, bits, group, kind, 5))


@pytest.mark.parametrize("bits,kind,group", KINDS)
@pytest.mark.parametrize("call", ["quantize_a8", "dequant", "codes", "gemv", "gemm", "gemv_a8", "gemm_a8", "grouped"])
def test_outputs_of_another_stream_are_not_what_this_one_still_writes(gpu, call, bits, kind, group):
    """Tensors that the current stream has yet to fill are dropped just before a call on another stream
    allocates outputs of their sizes: those are written once, by the call."""
    import torch
    n, k, m = 512, 512, 64
    w = weight_of(gpu, bits, kind, group, n, k)
    experts = gpu.PackedExperts.stack([w, w])
    x, off = to_dev(activations(k, 6, m)), to_dev(np.array([0, 20, m], np.int32))
    xq, sx = gpu.quantize_a8(x)
    calls = {"quantize_a8": lambda s: gpu.quantize_a8(x, stream=s), "dequant": lambda s: w.dequant(stream=s),
             "codes": lambda s: w.dequant(gpu.QX_OUT_CODES, stream=s), "gemv": lambda s: w.gemv(x[0], stream=s),
             "gemm": lambda s: w.gemm(x, stream=s), "gemv_a8": lambda s: w.gemv_a8(x[0], stream=s),
             "gemm_a8": lambda s: w.gemm_a8(xq, sx, stream=s), "grouped": lambda s: experts.gemm(x, off, stream=s)}

    def outputs(s):
        y = calls[call](s)
        return y if isinstance(y, tuple) else (y,)

    want = [t.clone() for t in outputs(None)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        torch.cuda._sleep(20_000_000)
        dropped = [torch.empty_like(t).fill_(3) for t in want]
        del dropped
        got = outputs(other)
        other.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))


def test_a_product_of_a_dropped_quantization_on_a_stream(gpu):
    """Rows that were quantized on a stream are dropped while a product of that stream still has to read
    them, and the current stream takes memory of their size: the product is the eager one."""
    import torch
    n, k, m = 300, 1024, 70
    w = weight_of(gpu, 3, 0, 64, n, k)
    x = to_dev(activations(k, 6, m))
    want = w.gemm_a8(*gpu.quantize_a8(x)).clone()
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(other):
            torch.cuda._sleep(20_000_000)
        xq, sx = gpu.quantize_a8(x, stream=other)
        y = w.gemm_a8(xq, sx, stream=other)
        shape = xq.shape
        del xq, sx
        torch.full(shape, 7, dtype=torch.int8, device="cuda")
        torch.full((m,), 3.0, device="cuda")
        torch.cuda.synchronize()
        assert torch.equal(y, want)
