"""Attention calls on both sides of the sizes from which work is shared out instead of a block an item, over both caches, against 64 bits."""
import pytest
import torch

import test_gpu_kv4 as four
import test_gpu_kv8 as eight

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    c = Context()
    yield c
    c.close()


def _both(ctx, bits, *args, **kw):
    if bits == 4:
        four._attend(ctx, *args, **kw)
    else:
        eight._attend(ctx, "e4m3", *args, **kw)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("longest", [32, 512, 513, 1024, 1025])
@pytest.mark.parametrize("new", [1, 3, 5])
def test_few_rows(ctx, bits, longest, new):
    _both(ctx, bits, [longest - new, 0, 7, 130], [new, 1, 0, new], 2, 4, 32, 64)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("longest", [300, 1100])
def test_more_requests_than_are_looked_at_at_once(ctx, bits, longest):
    past = [5, 40, 0] * 45
    new = [1, 0, 2] * 45
    past[70] = longest
    _both(ctx, bits, past, new, 1, 4, 16, 64)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("past,new", [([0], [1024]), ([1], [1024]), ([924], [100]), ([925], [100]), ([500, 0, 90], [30, 0, 200])])
@pytest.mark.parametrize("window", [0, 200])
def test_prompts(ctx, bits, past, new, window):
    _both(ctx, bits, past, new, 2, 2, 32, 64, window=window)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("requests", [20, 150])
def test_a_prompt_among_single_tokens(ctx, bits, requests):
    """150: more row tiles that no request has than a block each is worth."""
    _both(ctx, bits, [9] * requests + [20], [1] * requests + [600], 2, 4, 16, 64)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("new", [1, 3, 40])
def test_pages_that_do_not_exist(ctx, bits, new):
    """An item of its own with a page outside the cache: reported, finite, and the other requests' rows as without it."""
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, Kv4Cache, Kv8Cache, SbError
    torch.manual_seed(0)
    lens = torch.tensor([new + 40, new + 90], dtype=torch.int32, device="cuda")
    starts, every = torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda"), torch.tensor([0, new + 40, 2 * new + 130], dtype=torch.int32, device="cuda")
    table = torch.arange(18, dtype=torch.int32, device="cuda").view(2, 9)
    x, q = torch.randn(2 * new + 130, 2, 64, device="cuda").bfloat16(), torch.randn(2 * new, 4, 64, device="cuda").bfloat16()
    cache = (Kv4Cache if bits == 4 else Kv8Cache).empty(18, 2, 16, 64, table)
    append, attention = (ctx.kv4_append, ctx.kv4_attention) if bits == 4 else (ctx.kv8_append, ctx.kv8_attention)
    append(cache, x, x, every, lens, new + 90)
    want, _ = attention(cache, q, starts, lens, new, new + 90)
    ctx.sync()
    table[0, 1] = 18
    got, _ = attention(cache, q, starts, lens, new, new + 90)
    with pytest.raises(SbError) as e:
        ctx.sync()
    assert e.value.status == SB_ERR_INVALID
    assert torch.equal(got[new:], want[new:]) and torch.isfinite(got).all()
