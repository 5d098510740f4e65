"""4-bit quantisation with a tensor scale far too small for the data: block scales and codes end at their largest number."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref
from test_gpu_fp4 import DEV, _quantise, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size,g", [(2.0 ** 100, 2.0 ** -40), (2.0 ** 127, 2.0 ** -120), (2.0 ** 60, 2.0 ** -100), (2.0 ** 127, 1.0),
                                    (2.0 ** 20, 2.0 ** -149), (3e38, 0.0371)])
def test_quotients_beyond_the_end_of_fp32(ctx, size, g):  # noqa: F811
    rng = np.random.default_rng(3)
    x = ref.bf16(rng.uniform(-1, 1, (37, 200)) * size)
    x[5, 16:32] = 0                                        # a block of zeros keeps scale 0
    x[6, 0] = 0
    x[7, 48], x[9, 60] = np.inf, np.nan
    m = _quantise(ctx, x, "nv", g)
    y = ctx.fp4_dequantize(m).double().cpu().numpy()
    ctx.sync()
    # the definition: s = e4m3 of (amax / 6) / g, at most 448; d = s g; codes of x / d, at most 6 in magnitude
    v = np.zeros((37, 224))
    v[:, :200] = x
    v = v.reshape(37, -1, 16)
    g32 = float(np.float32(g))
    bad = ~np.isfinite(v).all(-1)
    t = np.abs(np.where(np.isfinite(v), v, 0)).max(-1) / 6 / g32
    s = np.where(t > 448, 448.0, ref.round_e4m3(np.minimum(t, 448)))
    byte = ref.e4m3_bytes(s).copy()
    byte[bad] = 0x7f
    np.testing.assert_array_equal(m.scales.cpu().numpy(), ref.tiled_scales(byte))
    d = s * g32
    q = np.where((d == 0)[..., None] | bad[..., None], 0, v / np.where(d > 0, d, 1)[..., None])
    code = ref.round_e2m1(q.clip(-8, 8)).reshape(37, -1)
    got = m.codes.cpu().numpy()
    keep = ~np.repeat(bad, 16, axis=1)
    got = np.stack((got & 15, got >> 4), -1).reshape(37, -1)
    np.testing.assert_array_equal(np.where(keep, got, 0), np.where(keep, code, 0))
    want = ref.E2M1[code & 7] * np.where(code > 7, -1.0, 1.0) * np.repeat(d, 16, axis=1)
    want = torch.from_numpy(want[:, :200]).to(torch.float32).to(torch.bfloat16).double().numpy()
    keep = keep[:, :200]
    assert np.isnan(y[~keep]).all()
    np.testing.assert_array_equal(y[keep], want[keep])
