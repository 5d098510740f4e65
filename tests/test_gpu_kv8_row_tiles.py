"""Attention of items that fill one of a block's two row tiles, both, or one after the other in the same share."""
import pytest

from test_gpu_kv8 import KINDS, _attend, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past,new,heads,group,dim,window", [
    ([6000], [20], 1, 4, 128, 0), ([3000, 100, 1500, 0], [20, 60, 33, 5], 2, 4, 128, 0), ([200] * 12, [30, 40, 8, 64] * 3, 4, 4, 64, 0),
    ([900, 5000, 10], [128, 129, 257], 1, 1, 96, 0), ([4000, 2000], [33, 32], 2, 4, 128, 1000), ([130] * 40, [7, 33] * 20, 8, 4, 64, 0)])
def test_one_row_tile_and_two(ctx, kind, past, new, heads, group, dim, window):  # noqa: F811
    _attend(ctx, kind, past, new, heads, group, 16, dim, window=window)
