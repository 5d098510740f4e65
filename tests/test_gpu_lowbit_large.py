"""The forms of the 4-bit and cache kernels that only large or unusual calls take: several tiles for a pair of CTAs, four column
segments, four pieces a thread, prompts of several requests with wide heads, prompts in a graph."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref
from test_gpu_fp4 import DEV, FORMATS, _product, ctx  # noqa: F401  (ctx: the fixture)
from test_gpu_kv8 import KINDS, _attend, _cache, _device, _ints, _starts, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(2100, 5000, 300), (2100, 5000, 1100),     # 180 tiles of 256 x 256 for 74 pairs: three in a row
                                   (300, 300, 8256)])                           # four tiles: four segments of the columns
def test_products_of_many_tiles_or_segments(ctx, fmt, M, N, K):  # noqa: F811
    _product(ctx, M, N, K, fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("ld", [4100, 4112, 4101])
def test_a_large_matrix_is_its_rows(ctx, fmt, ld):  # noqa: F811
    """9601 x 4100 (40M elements: four pieces a thread, the last row tile of one row) against calls on slices of 1280
    rows (one piece a thread), and a sample of rows against the plain form."""
    from paper_2602_17698_b200.binding import Fp4Matrix
    rows, cols = 9601, 4100
    gen = torch.Generator(device=DEV).manual_seed(5)
    x = torch.empty(rows, 4104, dtype=torch.bfloat16, device=DEV)[:, :cols]
    x.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * torch.randn(cols, generator=gen, device=DEV).exp())
    g = None if fmt == "mx" else torch.tensor([0.0371], device=DEV)
    m = ctx.fp4_quantize(x, Fp4Matrix.empty(rows, cols, fmt, g, DEV))
    buf = torch.full((rows, ld), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.fp4_dequantize(m, buf[:, :cols])
    tile_bytes = m.scales.numel() // -(-rows // 128)
    for r0 in range(0, rows, 1280):
        r1 = min(rows, r0 + 1280)
        part = ctx.fp4_quantize(x[r0:r1], Fp4Matrix.empty(r1 - r0, cols, fmt, g, DEV))
        assert torch.equal(part.codes, m.codes[r0:r1])
        assert torch.equal(part.scales, m.scales[r0 // 128 * tile_bytes:][:part.scales.numel()])
        assert torch.equal(ctx.fp4_dequantize(part), buf[r0:r1, :cols])
    ctx.sync()
    assert (buf[:, cols:] == 7).all()
    pick = np.r_[0, 1, 127, 128, np.random.default_rng(1).integers(0, rows, 40), rows - 1]
    codes, _, d = ref.fp4_quantize(x[pick].float().cpu().numpy(), fmt, None if fmt == "mx" else 0.0371)
    np.testing.assert_array_equal(m.codes[pick].cpu().numpy(), codes)
    np.testing.assert_array_equal(buf[pick, :cols].float().cpu().numpy(), ref.bf16(ref.fp4_values(codes, d, cols).astype(np.float32)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past,new,group,dim,window", [([60, 0, 200], [30, 45, 1], 3, 256, 0), ([0, 90], [50, 33], 2, 144, 40), ([10, 11], [20, 0], 8, 208, 0)])
def test_prompts_with_wide_heads(ctx, kind, past, new, group, dim, window):  # noqa: F811
    _attend(ctx, kind, past, new, 2, group, 32, dim, window=window)


def test_prompts_in_a_graph():
    """A captured chunk of prompts replayed while the requests grow, against the same calls made one by one."""
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    rng = np.random.default_rng(3)
    heads, dim, page, new = 2, 128, 16, [60, 33]
    cache = _cache("e4m3", [2000, 700], heads, page, dim, rng)
    x, q = _device(_tokens(sum(new), heads, dim, rng)), _device(_tokens(sum(new), 8, dim, rng))
    starts, lens = _ints(_starts(new)), _ints([100, 33])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = Context(stream=side)
        dev, dev2 = cache.device(DEV), cache.device(DEV)
        out = torch.empty(sum(new), 8, dim, dtype=torch.bfloat16, device=DEV)
        c.kv8_attention(dev, q, starts, lens, 60, 2000, out=out)         # the workspace grows outside the capture
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.kv8_append(dev, x, x, starts, lens, 60)
            c.kv8_attention(dev, q, starts, lens, 60, 2000, out=out)
        for _ in range(10):
            lens += 61
            graph.replay()
            c.kv8_append(dev2, x, x, starts, lens, 60)
            want, _ = c.kv8_attention(dev2, q, starts, lens, 60, 2000)
            c.sync()
            assert torch.equal(out, want)
        del graph
        c.close()
