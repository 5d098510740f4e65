"""Attention over the 8-bit cache under any softmax scale: negative ones, on both sides of the number of query rows that
chooses the kernel."""
import pytest

from test_gpu_kv8 import KINDS, _attend, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


# The tolerances are _attend's: the sign of the scale changes no rounding, and its bounds take magnitudes. With scale -1 the
# scores of a block of 16 keys spread over some 40 powers of two.
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale", [-0.1, -1.0, -0.0])
@pytest.mark.parametrize("past,new,heads,group,dim,window", [
    ([200, 31], [1, 1], 2, 4, 128, 0), ([150, 0], [7, 6], 1, 4, 128, 0), ([200, 0, 33], [40, 70, 1], 1, 4, 128, 0),
    ([300], [33], 2, 2, 64, 50), ([100], [90], 1, 3, 96, 0), ([70, 20], [20, 9], 1, 2, 256, 0)])
def test_negative_scales(ctx, kind, scale, past, new, heads, group, dim, window):  # noqa: F811
    _attend(ctx, kind, past, new, heads, group, 16, dim, window=window, scale=scale)
