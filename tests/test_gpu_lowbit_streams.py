"""Contexts on a stream of their own, called while torch's current stream is another."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref
from test_gpu_fp4 import DEV, _bf16, _quantise
from test_gpu_kv8 import _cache, _device, _ints, _tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def side():
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    stream = torch.cuda.Stream()
    c = Context(stream=stream)
    yield c
    c.close()


def _calls(c):
    rng = np.random.default_rng(1)
    a, b = (_quantise(c, _bf16(n, 512, rng), "mx") for n in (40, 96))
    cache = _cache("int8", [90, 70], 2, 16, 64, rng)
    dev = cache.device(DEV)
    starts, lens, q = _ints([0, 20, 50]), _ints([90, 70]), _device(_tokens(50, 8, 64, rng))
    torch.cuda.synchronize()
    return {"gemm": lambda: [c.fp4_gemm(a, b)], "gemm fp32": lambda: [c.fp4_gemm(a, b, out_dtype=torch.float32)],
            "dequantize": lambda: [c.fp4_dequantize(a)], "read": lambda: list(c.kv8_read(dev, starts, lens, 30, total=50)),
            "attention": lambda: list(c.kv8_attention(dev, q, starts, lens, 30, 90, want_lse=True))}


@pytest.mark.parametrize("which", ["gemm", "gemm fp32", "dequantize", "read", "attention"])
def test_outputs_belong_to_the_stream_that_writes_them(side, which):
    """The stream is busy when the call is made; the outputs are let go at once and torch's current stream takes memory of their
    sizes. What it writes there has to stay."""
    call = _calls(side)[which]
    want = call()
    side.sync()
    shapes = [(t.shape, t.dtype) for t in want]
    with torch.cuda.stream(side.stream):
        torch.cuda._sleep(50_000_000)                      # some 30 ms
    outs = call()
    del outs
    mine = [torch.full(shape, 7.0, dtype=dtype, device=DEV) for shape, dtype in shapes]
    torch.cuda.synchronize()
    for t in mine:
        assert (t == 7).all()
    # and the other way round: memory that the current stream has let go but still writes
    torch.cuda._sleep(50_000_000)
    late = [torch.full(shape, 7.0, dtype=dtype, device=DEV) for shape, dtype in shapes]
    del late
    again = call()
    torch.cuda.synchronize()
    for t, w in zip(again, want):
        assert torch.equal(t, w)
