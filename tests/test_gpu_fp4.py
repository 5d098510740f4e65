"""Microscaled 4-bit formats against a plain implementation: quantisation bit for bit, products in 64 bits."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMATS = ["mx", "nv"]


@pytest.fixture(scope="module")
def ctx():
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    c = Context()
    yield c
    c.close()


def _bf16(rows, cols, rng, spread=1.0):
    x = rng.standard_normal((rows, cols)) * np.exp(spread * rng.standard_normal(cols))
    return ref.bf16(x)


def _device(x, pad=0):
    """bf16 on the device, rows 16-byte aligned, `pad` extra columns of NaN behind them."""
    rows, cols = x.shape
    ld = -(-cols // 8) * 8 + pad
    t = torch.full((rows, ld), float("nan"), dtype=torch.bfloat16, device=DEV)
    t[:, :cols] = torch.from_numpy(x).to(torch.bfloat16).to(DEV)
    return t[:, :cols]


def _quantise(ctx, x, fmt, g=None, pad=0):
    from paper_2602_17698_b200.binding import Fp4Matrix
    ts = None if g is None else torch.tensor([g], dtype=torch.float32, device=DEV)
    m = Fp4Matrix.empty(*x.shape, fmt, ts, DEV)
    m.codes.fill_(0xff)
    m.scales.fill_(0xff)
    return ctx.fp4_quantize(_device(x, pad), m)


def _check(ctx, x, fmt, g=None, pad=0):
    m = _quantise(ctx, x, fmt, g, pad)
    ctx.sync()
    codes, byte, d = ref.fp4_quantize(x, fmt, g)
    np.testing.assert_array_equal(m.scales.cpu().numpy(), ref.tiled_scales(byte))
    got = m.codes.cpu().numpy()
    nan = np.repeat(np.isnan(d), (16 if fmt == "mx" else 8), axis=1)       # codes of a NaN block are any
    np.testing.assert_array_equal(np.where(nan, 0, got), np.where(nan, 0, codes))
    return m, codes, d


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 17), (2, 100), (127, 48), (128, 256), (130, 4100), (1000, 33), (5, 16384)])
def test_quantisation_is_exact(ctx, fmt, rows, cols):
    rng = np.random.default_rng(rows * 7 + cols)
    x = _bf16(rows, cols, rng)
    _check(ctx, x, fmt, None if fmt == "mx" else float(2.0 ** -7), pad=8 * (rows % 3))


@pytest.mark.parametrize("g", [None, 1.0, 0.0123, 3.7e-5, 2.0 ** -120, 1e30])
def test_any_tensor_scale(ctx, g):
    """Scales that are no power of two, and such small or large ones that the quotient is taken the long way."""
    rng = np.random.default_rng(5)
    x = ref.bf16(_bf16(40, 500, rng) * np.float32(500 * (g or 1.0)))
    _check(ctx, x, "nv", g)


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_bf16_number_and_ties(ctx, fmt):
    """All finite bf16 values as the largest of a block, against midpoints of the grid."""
    bits = np.arange(0, 0x7f80, 7, dtype=np.uint32)
    top = (bits << 16).view(np.float32)
    f = np.array([1, -1, .5, .25, -.75, 1 / 3, 0, -0.0, .875, .625, -.4375, .3125, .2083, .0417, .125, 1 / 24], dtype=np.float32)
    with np.errstate(all="ignore"):
        x = ref.bf16(np.concatenate([top[:, None] * f, top[:, None] * -f], 1))
    x = np.where(np.isfinite(x), x, 0)
    _check(ctx, x, fmt, None if fmt == "mx" else 1.0)


@pytest.mark.parametrize("fmt", FORMATS)
def test_not_a_number_and_infinity_stay_in_their_block(ctx, fmt):
    rng = np.random.default_rng(1)
    x = _bf16(9, 130, rng)
    x[0, 5], x[3, 70], x[8, 129], x[4, 40] = np.nan, np.inf, -np.inf, -np.nan
    x[6] = 0
    m, codes, d = _check(ctx, x, fmt, None if fmt == "mx" else 0.25)
    y = ctx.fp4_dequantize(m).float().cpu().numpy()
    ctx.sync()
    want = ref.bf16(ref.fp4_values(codes, d, 130))
    np.testing.assert_array_equal(np.isnan(y), np.isnan(want))
    np.testing.assert_array_equal(np.nan_to_num(y), np.nan_to_num(want))
    assert np.isnan(y[0, 5]) and not np.isnan(y[1]).any()


def test_a_tensor_scale_that_is_not_positive_gives_not_a_number(ctx):
    x = _bf16(2, 32, np.random.default_rng(1))
    for g in (0.0, -1.0, float("nan")):
        y = ctx.fp4_dequantize(_quantise(ctx, x, "nv", g))
        assert torch.isnan(y).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols,ld", [(1, 1, 1), (3, 17, 17), (5, 33, 40), (64, 128, 128), (130, 1000, 1001), (2, 15, 16)])
def test_dequantisation_rounds_once(ctx, fmt, rows, cols, ld):
    rng = np.random.default_rng(cols)
    x = _bf16(rows, cols, rng)
    g = None if fmt == "mx" else 0.0371
    m, codes, d = _check(ctx, x, fmt, g)
    buf = torch.full((rows, ld), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.fp4_dequantize(m, buf[:, :cols])
    ctx.sync()
    # block scale times code: exact in 64 bits, fp32 in between (d has at most 24 + 4 bits)
    want = ref.bf16((ref.fp4_values(codes, d, cols)).astype(np.float32))
    np.testing.assert_array_equal(buf[:, :cols].float().cpu().numpy(), want)
    assert (buf[:, cols:] == 7).all()


def _product(ctx, M, N, K, fmt, seed=0, ldy=None):
    rng = np.random.default_rng(seed + M + 3 * N + 7 * K)
    ga, gb = (None, None) if fmt == "mx" else (2.0 ** -6, 0.0173)
    a, b = _bf16(M, K, rng), _bf16(N, K, rng) * np.float32(0.05)
    b = ref.bf16(b)
    ma, mb = _quantise(ctx, a, fmt, ga), _quantise(ctx, b, fmt, gb)
    va = ref.fp4_values(*ref.fp4_quantize(a, fmt, ga)[::2], K)
    vb = ref.fp4_values(*ref.fp4_quantize(b, fmt, gb)[::2], K)
    buf = torch.full((M, ldy or N), float("nan"), dtype=torch.float32, device=DEV)
    y = ctx.fp4_gemm(ma, mb, out=buf[:, :N])
    ctx.sync()
    want, mag = va @ vb.T, np.abs(va) @ np.abs(vb).T
    # products of codes and scales are exact; the tensor cores add in fp32, each addition off by at
    # most 2^-23 of what it adds (they cut off instead of rounding), at most K / 16 additions in a
    # row, an error that grows like their square root: 2^-23 * sqrt(1024) = 4e-6 of the sum of
    # magnitudes; plus the tensor scales' product and the last rounding
    tol = 4e-6 * mag + 2.0 ** -22 * np.abs(want) + 1e-30
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
    # the same sums in bf16: rounded once
    low = torch.full((M, ldy or N), float("nan"), dtype=torch.bfloat16, device=DEV)
    assert torch.equal(ctx.fp4_gemm(ma, mb, out=low[:, :N]), y.to(torch.bfloat16))
    assert torch.isnan(buf[:, N:]).all() and torch.isnan(low[:, N:]).all()
    return y


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(1, 128, 64), (1, 1, 1), (1, 128, 256), (16, 128, 1024), (7, 130, 96), (17, 64, 320), (33, 257, 4096),
                                   (64, 128, 32), (65, 384, 512), (128, 128, 2048), (129, 500, 1000), (300, 300, 300),
                                   (513, 1000, 768), (260, 4096, 512), (1000, 129, 4100)])
def test_product(ctx, fmt, M, N, K):
    _product(ctx, M, N, K, fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K,ldy", [(5, 100, 512, 101), (200, 130, 640, 131), (1, 4096, 4096, 4096), (700, 515, 1280, 517)])
def test_product_into_rows_of_any_length(ctx, fmt, M, N, K, ldy):
    _product(ctx, M, N, K, fmt, ldy=ldy)


@pytest.mark.parametrize("M", [1, 20, 500])
def test_product_is_the_same_every_time(ctx, M):
    one, two = (_product(ctx, M, 640, 2048, "nv") for _ in range(2))
    assert torch.equal(one, two)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M", [3, 200, 600])
def test_not_a_number_reaches_its_row_and_column_only(ctx, fmt, M):
    rng = np.random.default_rng(2)
    a, b = _bf16(M, 256, rng), _bf16(300, 256, rng)
    a[1, 100], b[130, 17] = np.nan, np.inf
    y = ctx.fp4_gemm(_quantise(ctx, a, fmt), _quantise(ctx, b, fmt))
    ctx.sync()
    nan = torch.isnan(y).cpu().numpy()
    want = np.zeros_like(nan)
    want[1], want[:, 130] = True, True
    np.testing.assert_array_equal(nan, want)


def test_on_another_stream_and_in_a_graph(ctx):
    from paper_2602_17698_b200.binding import Context, Fp4Matrix
    rng = np.random.default_rng(3)
    x, w = _bf16(4, 512, rng), _bf16(256, 512, rng)
    xd, m = _device(x), Fp4Matrix.empty(4, 512, "nv", None, DEV)
    mw = _quantise(ctx, w, "nv")
    want = ctx.fp4_gemm(_quantise(ctx, x, "nv"), mw)
    ctx.sync()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = Context(stream=side)
        y = torch.zeros(4, 256, dtype=torch.bfloat16, device=DEV)
        other.fp4_gemm(other.fp4_quantize(xd, m), mw, out=y)
        other.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            other.fp4_gemm(other.fp4_quantize(xd, m), mw, out=y)
        y.zero_()
        graph.replay()
        other.sync()
        assert torch.equal(y, want)
        del graph
        other.close()


def test_refusals(ctx):
    from paper_2602_17698_b200.binding import Fp4Matrix, SB_ERR_INVALID, SB_ERR_SHAPE, SbError, lib
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    m, g = Fp4Matrix.empty(4, 64, "mx", None, DEV), torch.ones(1, device=DEV)
    launches = ctx.kernel_launches()
    for status, call in [
        (SB_ERR_SHAPE, lambda: ctx.fp4_quantize(torch.zeros(4, 65, dtype=torch.bfloat16, device=DEV)[:, 1:], m)),
        (SB_ERR_INVALID, lambda: ctx.fp4_quantize(x, Fp4Matrix(m.codes, m.scales, 4, 64, "mx", g))),
        (SB_ERR_INVALID, lambda: ctx.fp4_dequantize(Fp4Matrix(m.codes, m.scales, 4, 64, "mx", g))),
        (SB_ERR_INVALID, lambda: ctx.fp4_gemm(Fp4Matrix(m.codes, m.scales, 4, 64, "mx", g), m)),
    ]:
        with pytest.raises(SbError) as e:
            call()
        assert e.value.status == status
    for call in [lambda: Fp4Matrix(m.codes, m.scales, 4, 65, "mx"), lambda: Fp4Matrix(m.codes, m.scales, 4, 64, "e5m2"),
                 lambda: Fp4Matrix(m.codes[:, :8], m.scales, 4, 64, "mx"), lambda: ctx.fp4_quantize(x[:3], m),
                 lambda: ctx.fp4_gemm(m, Fp4Matrix.empty(4, 64, "nv", None, DEV)), lambda: ctx.fp4_gemm(m, Fp4Matrix.empty(4, 96, "mx", None, DEV)),
                 lambda: ctx.fp4_gemm(m, m, out=torch.zeros(4, 4, dtype=torch.float16, device=DEV)),
                 lambda: ctx.fp4_dequantize(m, torch.zeros(4, 63, dtype=torch.bfloat16, device=DEV))]:
        with pytest.raises((ValueError, TypeError)):
            call()
    h, L = ctx._h, lib()
    c, s, p = m.codes.data_ptr(), m.scales.data_ptr(), x.data_ptr()
    assert L.sb_fp4_quantize(h, None, 4, 64, 64, 0, None, c, s) == SB_ERR_INVALID
    assert L.sb_fp4_quantize(h, p, 0, 64, 64, 0, None, c, s) == SB_ERR_INVALID
    assert L.sb_fp4_quantize(h, p, 4, 64, 64, 2, None, c, s) == SB_ERR_INVALID
    assert L.sb_fp4_quantize(h, p, 4, 64, 56, 0, None, c, s) == SB_ERR_SHAPE
    assert L.sb_fp4_quantize(h, p, 4, 64, 64, 0, None, c + 8, s) == SB_ERR_SHAPE
    assert L.sb_fp4_dequantize(h, c, s, 4, 64, 0, None, p, 63) == SB_ERR_SHAPE
    assert L.sb_fp4_gemm(h, c, s, None, 4, c, s, None, 4, 64, 0, p, 0, 3) == SB_ERR_SHAPE
    assert L.sb_fp4_gemm(h, c, s, None, 4, c, s, None, 4, 64, 0, p + 2, 1, 4) == SB_ERR_SHAPE
    assert L.sb_fp4_gemm(h, c, s, None, 0, c, s, None, 4, 64, 0, p, 0, 4) == SB_ERR_INVALID
    assert L.sb_fp4_gemm(None, c, s, None, 4, c, s, None, 4, 64, 0, p, 0, 4) == SB_ERR_INVALID
    assert ctx.kernel_launches() == launches
    ctx.sync()
