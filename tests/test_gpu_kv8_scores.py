"""Attention over the 8-bit cache where the running maximum of a row has to move, or must not."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref
from test_gpu_kv8 import DEV, KINDS, _attend, _cache, _ints, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


def _ramp(way):
    """Key scales that rise or fall from block to block of a request (so do its scores' sizes), or that
    are the same for all keys, whose codes are then made the same too."""
    def change(cache):
        blocks = cache.scale[0].shape[2]
        for row in cache.table:
            for i, pg in enumerate(row):
                for j in range(blocks):
                    at = i * blocks + j
                    f = {"rise": 1.02 ** at, "fall": 0.98 ** at, "steps": 1 + at // 9 % 2 * 3.0, "same": 1.0}[way]
                    cache.scale[0][pg, :, j] = ref.bf16(cache.scale[0][pg, :, j] * f)
        if way == "same":
            cache.scale[0][:] = ref.bf16(np.full(cache.scale[0].shape, 0.01))
            cache.code[0][:] = cache.code[0][cache.table[0, 0], :, 0][None, :, None, :]
    return change


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("way", ["rise", "fall", "steps", "same"])
@pytest.mark.parametrize("past,new,group,dim,qsize", [
    ([1100], [1], 4, 128, 1.0), ([1100, 500], [70, 40], 4, 128, 1.0), ([1100], [70], 4, 64, 4.0), ([700], [3], 8, 64, 4.0),
    ([0], [300], 1, 128, 2.0)])
def test_scores_that_rise_and_fall(ctx, kind, way, past, new, group, dim, qsize):  # noqa: F811
    _attend(ctx, kind, past, new, 1, group, 16, dim, qsize=qsize, change=_ramp(way), poison=False)


@pytest.mark.parametrize("group", [1, 4, 8])
@pytest.mark.parametrize("new", [2, 3, 4, 6, 7, 24, 25, 26])
def test_both_sides_of_the_row_counts_that_choose_the_kernel(ctx, group, new):  # noqa: F811
    _attend(ctx, "int8", [150, 0, 33], [new, 1, new - 1], 2, group, 32, 128)


@pytest.mark.parametrize("requests,past,new", [(1, 2000, 1), (3, 190, 3), (5, 7, 2), (2, 600, 2)])
def test_shares_smaller_than_an_item(ctx, requests, past, new):  # noqa: F811
    _attend(ctx, "e4m3", [past + 16 * b for b in range(requests)], [new] * requests, 4, 4, 16, 128)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("new", [1, 40])
def test_a_query_that_is_no_number_stays_in_its_row(ctx, bad, new):  # noqa: F811
    rng = np.random.default_rng(new)
    cache = _cache("int8", [300 + new], 1, 16, 128, rng)
    dev = cache.device(DEV)
    q = torch.from_numpy(ref.bf16(rng.standard_normal((new, 4, 128)))).to(torch.bfloat16).to(DEV)
    want, _, mag, top, held = ref.attention(cache, q.double().cpu().numpy(), [0, new], [300 + new], 0.1, 0)
    q[new // 2, 1, 5] = bad
    got, _ = ctx.kv8_attention(dev, q, _ints([0, new]), _ints([300 + new]), new, 300 + new, scale=0.1)
    ctx.sync()
    got = got.double().cpu().numpy()
    assert np.isnan(got[new // 2, 1]).any()
    # every other row as ever: the result's rounding, the weights', the scores' sums (see _attend)
    eps = 2.0 ** -20 * (top + 1)
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * eps[..., None]) * mag + 2.0 ** -24 * held + 1e-30
    keep = np.ones((new, 4), bool)
    keep[new // 2, 1] = False
    assert (np.abs(got - want) <= tol)[keep].all()
