"""Attention where the value scales of a request's blocks lie far apart, and the small ones carry the result."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref
from test_gpu_kv8 import DEV, KINDS, _cache, _device, _ints, _starts, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ratio", [2.0 ** 10, 2.0 ** 18, 2.0 ** 21, 2.0 ** 60])
@pytest.mark.parametrize("past,new,group,dim", [([400, 70], [1, 1], 4, 128), ([300], [5], 4, 64), ([400, 60], [40, 33], 4, 128), ([200], [90], 2, 64)])
def test_a_block_of_large_values_that_nobody_looks_at(ctx, kind, ratio, past, new, group, dim):  # noqa: F811
    """The first block's values are `ratio` times the others', but its keys' weights are next to nothing."""
    rng = np.random.default_rng(sum(past) + dim)
    lens, starts, scale = [p + n for p, n in zip(past, new)], _starts(new), dim ** -0.5
    cache = _cache(kind, lens, 1, 16, dim, rng)
    q = ref.bf16(rng.standard_normal((starts[-1], group, dim)) * 0.25)
    q[..., 0] = 8.0
    for row in cache.table:
        cache.scale[1][row[0]] = ref.bf16(cache.scale[1][row[0]] * ratio)
        # keys of the first block: 100 / scale against the queries' first element, some e^-100 of the others' weights
        cache.scale[0][row[0]] = ref.bf16(np.full(1, 100 / (scale * 8 * 100)))
        cache.code[0][row[0]] = 0
        cache.code[0][row[0], :, :, 0] = -100 if kind == "int8" else -104
    out, _ = ctx.kv8_attention(cache.device(DEV), _device(q), _ints(starts), _ints(lens), max(new), max(lens), scale=scale)
    ctx.sync()
    want, _, mag, top, _ = ref.attention(cache, q, starts, lens, scale, 0)
    # the last rounding 2^-8 of the result, the weights' 2^-11 of weight x |v|, the scores' sums 2^-20 of their terms: no term
    # under the largest value scale, since a weight times its value scale is held relative to what the row's keys add
    eps = 2.0 ** -20 * (top + 1)
    # (the scores of rows that do see the others: all but those whose keys all lie in the first block)
    seen = np.concatenate([np.arange(ln - n, ln) >= 16 for ln, n in zip(lens, new)])
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * eps[..., None]) * mag + 1e-30
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= tol)[seen].all(), float((err / tol)[seen].max())
