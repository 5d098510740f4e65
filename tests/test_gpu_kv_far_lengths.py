"""Requests of up to 2^31 - 65536 tokens, all of one page that the table repeats: keys of zeros, so that every weight is the same, and values of
which each token has one element, so that the sums are exact and the log-sum-exp is the log of how many keys a query sees."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, PAGE, MOST = "cuda:0", 16, (1 << 31) - 65536


@pytest.fixture(scope="module")
def ctx():
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    c = Context()
    yield c
    c.close()


@pytest.fixture(scope="module")
def table():
    t = torch.zeros(1, (1 << 31) // PAGE - 1, dtype=torch.int32, device=DEV)
    yield t
    del t
    torch.cuda.empty_cache()


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _cache(ctx, bits, table):
    """One page: token t has value 1 in element t."""
    from paper_2602_17698_b200.binding import Kv4Cache, Kv8Cache
    cache = (Kv4Cache if bits == 4 else Kv8Cache).empty(1, 1, PAGE, 16, table)
    k, v = torch.zeros(PAGE, 1, 16, dtype=torch.bfloat16, device=DEV), torch.eye(16, device=DEV).bfloat16()[:, None].contiguous()
    (ctx.kv4_append if bits == 4 else ctx.kv8_append)(cache, k, v, _ints(0, PAGE), _ints(PAGE), PAGE)
    ctx.sync()
    return cache, ctx.kv4_attention if bits == 4 else ctx.kv8_attention


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("new,length,window", [(1, MOST, 0), (3, MOST, 0), (1, MOST - 16 * 5, 0), (2, MOST, 3 << 29), (1, MOST, MOST - 16), (40, MOST, 1 << 20),
                                               (300, MOST, 5000), (1, MOST, 100)])
def test_attention_near_the_limit(ctx, table, bits, new, length, window):
    cache, attention = _cache(ctx, bits, table)
    q = torch.randn(new, 1, 16, device=DEV).bfloat16()
    out, lse = attention(cache, q, _ints(0, new), _ints(length), new, length, window=window, want_lse=True)
    ctx.sync()
    for i in range(new):
        p = length - new + i
        keys = min(p + 1, window) if window else p + 1
        assert abs(float(lse[i, 0]) - math.log(keys)) <= 2.0 ** -20 * math.log(keys)
    # 4 bits hold 1 as 6 x 1.375 / 8 = 1.03125: its scale 1 / 6 rounded to e4m3, whose steps there are 1 / 64, and the code of 1 / 0.171875 = 5.8
    value = 1.03125 if bits == 4 else 1.0
    # a value is one of PAGE equal weights (but for the ragged rest of a window); 8 bits: its scale, rounded up to bf16, times 127 (2^-8), and a weight in
    # fp16 (2^-11); the result's rounding. A warp adds up to 2^31 / 32 / 4 / 148 steps of two products of 16 keys each, a bit of 2^-23 lost at each
    steps = 2 * (min(length, window or length) / 32 / 4 / 148 + 1)
    rest = PAGE / min(length - new + 1, window or length)
    assert float((out.float() - value / PAGE).abs().max()) <= value * (2.0 ** -8 + (0 if bits == 4 else 2.0 ** -8 + 2.0 ** -11 + steps * 2.0 ** -23) + rest) / PAGE


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("length", [MOST + 1, (1 << 31) - 16])
def test_longer_requests_are_skipped_and_reported(ctx, table, bits, new, length):
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SbError
    cache, attention = _cache(ctx, bits, table)
    x = torch.ones(new, 1, 16, dtype=torch.bfloat16, device=DEV)
    held = [t.clone() for t in (cache.k, cache.v)]
    for call in ("append", "read", "attention"):
        out = [torch.full_like(x, 7.0) for _ in range(2)]
        if call == "append":
            (ctx.kv4_append if bits == 4 else ctx.kv8_append)(cache, x, x, _ints(0, new), _ints(length), new)
        elif call == "read":
            (ctx.kv4_read if bits == 4 else ctx.kv8_read)(cache, _ints(0, new), _ints(length), new, out=out)
        else:
            attention(cache, x, _ints(0, new), _ints(length), new, length, out=out[0])
        with pytest.raises(SbError) as e:
            ctx.sync()
        assert e.value.status == SB_ERR_INVALID
        assert all((o == 7).all() for o in out)
        assert torch.equal(cache.k.view(torch.uint8), held[0].view(torch.uint8)) and torch.equal(cache.v.view(torch.uint8), held[1].view(torch.uint8))
