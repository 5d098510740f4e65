"""Attention whose workspaces grow while a graph is captured (a capture that allows allocations)."""
import ctypes

import numpy as np
import pytest
import torch

from test_gpu_kv8 import DEV, _cache, _device, _ints, _starts, _tokens

pytestmark = pytest.mark.gpu


def _dirty():
    """Memory that was in use and is free again: what the next small allocations get is not zero."""
    rt = ctypes.CDLL("libcudart.so.12")
    torch.cuda.synchronize()
    held = []
    for size in [20_000] * 300 + [1 << 20] * 8:
        p = ctypes.c_void_p()
        assert rt.cudaMalloc(ctypes.byref(p), ctypes.c_size_t(size)) == 0
        assert rt.cudaMemset(p, 0x5a, ctypes.c_size_t(size)) == 0
        held.append(p)
    torch.cuda.synchronize()
    for p in held:
        assert rt.cudaFree(p) == 0


@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
def test_a_first_call_inside_a_capture(new):
    """What the capture allocated is ready for calls outside of the graph, before its first replay and after."""
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    rng = np.random.default_rng(3)
    heads, dim = 2, 128
    cache = _cache("int8", [4000, 700], heads, 16, dim, rng)
    q, starts, lens = _device(_tokens(sum(new), 8, dim, rng)), _ints(_starts(new)), _ints([3500, 700])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        plain, c = Context(stream=side), Context(stream=side)
        dev = cache.device(DEV)
        want, _ = plain.kv8_attention(dev, q, starts, lens, max(new), 4000)
        plain.sync()
        out = torch.zeros_like(want)
        _dirty()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side, capture_error_mode="relaxed"):
            c.kv8_attention(dev, q, starts, lens, max(new), 4000, out=out)
        got = torch.zeros_like(want)
        c.kv8_attention(dev, q, starts, lens, max(new), 4000, out=got)
        c.sync()
        assert torch.equal(got, want)
        graph.replay()
        c.kv8_attention(dev, q, starts, lens, max(new), 4000, out=got.zero_())
        c.sync()
        assert torch.equal(out, want) and torch.equal(got, want)
        del graph
        plain.close()
        c.close()
