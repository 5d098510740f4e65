"""Caches whose page table is part of a wider one, or one row for all requests."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref
from test_gpu_kv8 import DEV, KINDS, _cache, _device, _ints, _same, _starts, _tokens, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


def _with_table(dev, table):
    from paper_2602_17698_b200.binding import Kv8Cache
    return Kv8Cache(dev.k, dev.v, dev.k_scale, dev.v_scale, table)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [[1, 1, 1], [20, 3, 40]])
def test_rows_of_a_wider_table(ctx, kind, new):  # noqa: F811
    """The same results, and the entries behind a request's own are not its pages, whichever pages they name."""
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SbError
    rng = np.random.default_rng(sum(new))
    heads, dim, page, lens = 2, 64, 16, [60, 33, 64]
    cache = _cache(kind, [64, 64, 64], heads, page, dim, rng, spare=4)
    dev = cache.device(DEV)
    spare = sorted(set(range(cache.code[0].shape[0])) - set(cache.table.ravel()))
    wide = torch.tensor(spare[:2], dtype=torch.int32, device=DEV).repeat(3, 3)
    wide[:, :4] = dev.table
    part = _with_table(dev, wide[:, :4])
    starts = _starts(new)
    x, q = _tokens(starts[-1], heads, dim, rng), _device(_tokens(starts[-1], 4 * heads, dim, rng))
    ctx.kv8_append(part, _device(x), _device(x), _ints(starts), _ints(lens), max(new))
    for side in range(2):
        cache.append(side, x, starts, lens)
    got = ctx.kv8_attention(part, q, _ints(starts), _ints(lens), max(new), 64, want_lse=True)
    want = ctx.kv8_attention(dev, q, _ints(starts), _ints(lens), max(new), 64, want_lse=True)
    back = ctx.kv8_read(part, _ints(starts), _ints(lens), max(new), total=starts[-1])
    ctx.sync()
    _same(cache, dev)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.isfinite(back[0].float()).all()
    # one token more than the row's four pages hold, though the wider table goes on: skipped and reported, in every row
    for b in range(3):
        longer = list(lens)
        longer[b] = 65
        for call in (lambda: ctx.kv8_append(part, _device(x), _device(x), _ints(starts), _ints(longer), max(new)),
                     lambda: ctx.kv8_attention(part, q, _ints(starts), _ints(longer), max(new), 65),
                     lambda: ctx.kv8_read(part, _ints(starts), _ints(longer), max(new), total=starts[-1])):
            call()
            with pytest.raises(SbError) as e:
                ctx.sync()
            assert e.value.status == SB_ERR_INVALID
    _same(cache, dev)                                       # the others' tokens are written again, and change nothing


@pytest.mark.parametrize("new", [[1, 1, 1], [30, 3, 7]])
def test_one_row_for_all_requests(ctx, new):  # noqa: F811
    """Requests that read the same pages, each up to a length of its own."""
    rng = np.random.default_rng(5)
    heads, dim, page, lens = 2, 128, 32, [200, 3, 77]
    cache = _cache("int8", [200], heads, page, dim, rng)
    dev = cache.device(DEV)
    starts = _starts(new)
    q = _device(_tokens(starts[-1], 4 * heads, dim, rng))
    got, gl = ctx.kv8_attention(_with_table(dev, dev.table.expand(3, -1)), q, _ints(starts), _ints(lens), max(new), 200, want_lse=True)
    want, wl = ctx.kv8_attention(_with_table(dev, dev.table.repeat(3, 1)), q, _ints(starts), _ints(lens), max(new), 200, want_lse=True)
    ctx.sync()
    assert torch.equal(got, want) and torch.equal(gl, wl)
