"""Values of 4-bit matrices written to rows of every alignment, next to memory that stays as it is."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref
from test_gpu_fp4 import DEV, FORMATS, _bf16, _check, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (7, 40), (33, 47), (9, 130), (40, 1000), (3, 4090)])
@pytest.mark.parametrize("base,pad", [(0, 0), (0, 1), (0, 2), (8, 8), (16, 16), (1, 0), (2, 6), (3, 5)])
def test_rows_of_any_alignment(ctx, fmt, rows, cols, base, pad):  # noqa: F811
    rng = np.random.default_rng(rows + cols)
    m, codes, d = _check(ctx, _bf16(rows, cols, rng), fmt, None if fmt == "mx" else 0.0371)
    ld = (-(-cols // pad) * pad if pad > 2 else cols + pad)
    buf = torch.full((base + rows * ld + 64,), 7.0, dtype=torch.bfloat16, device=DEV)
    out = buf[base:base + rows * ld].view(rows, ld)
    ctx.fp4_dequantize(m, out[:, :cols])
    ctx.sync()
    want = ref.bf16(ref.fp4_values(codes, d, cols).astype(np.float32))
    np.testing.assert_array_equal(out[:, :cols].float().cpu().numpy(), want)
    assert (out[:, cols:] == 7).all() and (buf[:base] == 7).all() and (buf[base + rows * ld:] == 7).all()
