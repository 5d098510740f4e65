"""Batches whose slots are mostly without tokens: the same results, and no CTA a slot where there are very many."""
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


def _attend(ctx, bits, *args, **kw):
    before = ctx.kernel_launches()
    if bits == 4:
        four._attend(ctx, *args, **kw)
    else:
        eight._attend(ctx, "int8", *args, **kw)
    return ctx.kernel_launches() - before


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("slots", [600, 6000])
@pytest.mark.parametrize("new,dim", [(1, 128), (3, 64), (1, 80)])
def test_few_rows(ctx, bits, slots, new, dim):
    """Both sides of the number of empty slots from which work is shared out."""
    past, tokens = [0] * slots, [0] * slots
    for at, p in ((0, 9), (slots // 2, 40), (slots - 1, 0)):
        past[at], tokens[at] = p, new
    _attend(ctx, bits, past, tokens, 2, 4, 16, dim, poison=False)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("slots,launches", [(200, 1), (3000, 3)])
def test_a_prompt(ctx, bits, slots, launches):
    """200: a CTA each, one launch; 3000: plan, shares and their sum."""
    past, tokens = [0] * slots, [0] * slots
    past[-1], tokens[-1] = 20, 100
    assert _attend(ctx, bits, past, tokens, 2, 2, 16, 64, poison=False) == launches
