"""Work shared out over CTAs (requests too long for a CTA each) with heads of every kind: as long as a kernel's tile, shorter, and every number of query rows a
kernel is made for; over both caches, against 64 bits."""
import pytest
import torch

import test_gpu_kv4 as four
import test_gpu_kv8 as eight

pytestmark = pytest.mark.gpu
STEP, TILE = 32, 128          # keys of a step (few rows) and of a tile (prompts)


@pytest.fixture(scope="module")
def ctx():
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    c = Context()
    yield c
    c.close()


def _attend(ctx, bits, *args, **kw):
    before = ctx.kernel_launches()
    if bits == 4:
        four._attend(ctx, *args, **kw)
    else:
        eight._attend(ctx, bits, *args, **kw)
    return ctx.kernel_launches() - before


@pytest.mark.parametrize("bits", [4, "int8", "e4m3"])
@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 96, 112, 128, 144, 208, 240, 256])
@pytest.mark.parametrize("new,group", [(1, 4), (1, 8), (3, 4), (2, 8), (5, 4), (3, 8)])
def test_few_rows(ctx, bits, dim, new, group):
    """4 to 24 query rows; the longest request has more steps than an item of its own may have."""
    past = [1301, 40, 0, 700]
    assert (max(past) + new + STEP - 1) // STEP + 1 > 33
    _attend(ctx, bits, past, [new, new, 1, 0], 1, group, 48, dim, poison=False)


@pytest.mark.parametrize("bits", [4, "int8", "e4m3"])
@pytest.mark.parametrize("dim", [48, 96, 128, 208])
@pytest.mark.parametrize("new,group", [(1, 5), (5, 4)])
def test_few_rows_in_a_window(ctx, bits, dim, new, group):
    """Shares of windows, whose first step starts inside a page; slots past the requests' ends hold NaN."""
    past, window = [1400, 1100], 1150
    assert (window + 8 + 16 + STEP - 1) // STEP + 1 > 33
    _attend(ctx, bits, past, [new, new], 2, group, 16, dim, window=window)


@pytest.mark.parametrize("bits", [4, "int8", "e4m3"])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 112, 128, 144, 208, 256])
@pytest.mark.parametrize("past,new,window", [([4200, 0], [90, 130], 0), ([5000, 60], [100, 81], 4300)])
def test_prompts(ctx, bits, dim, past, new, window):
    """More than 32 tiles of keys: plan, shares and their sum (8 bits with heads of more than 128: the kernel for few rows)."""
    assert (min(max(p + n for p, n in zip(past, new)), window or 1 << 30) + TILE - 1) // TILE > 32
    launches = _attend(ctx, bits, past, new, 1, 1, 16, dim, window=window, poison=False)
    assert launches == (1 if bits != 4 and dim > 128 else 3)
