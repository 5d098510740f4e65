"""Rotary positions against 64 bits."""
import numpy as np
import pytest
import torch

import lowbit_reference as low
import more_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def ctx():
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    c = Context()
    yield c
    c.close()


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def _rows(T, heads, dim, dtype, rng):
    x = torch.from_numpy(rng.standard_normal((T, heads, dim)).astype(np.float32)).to(dtype)
    return x.to(DEV), x.double().numpy()


def _table(rotated, interleaved, factor=1.0, base=10000.0, freq=None):
    from paper_2602_17698_b200.binding import RotaryTable, rotary_frequencies
    f = rotary_frequencies(rotated, base) if freq is None else torch.from_numpy(freq)
    return RotaryTable(f.to(DEV), interleaved, factor), f.numpy()


def _close(got, x, pos, freq, interleaved, factor, inverse, dtype):
    want, size = ref.rotary(x, pos, freq, interleaved, factor, inverse)
    # the result's rounding; cos and sin to two units of fp32 and the factor, 2^-22, both products and their sum, 2^-23, of both terms
    tol = HALF_STEP[dtype] * np.abs(want) + 2.0 ** -21 * size
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), (float((err / np.maximum(tol, 1e-300)).max()), np.unravel_index((err - tol).argmax(), err.shape))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rotated,hq,hk", [(128, 128, 32, 8), (64, 32, 4, 4), (80, 20, 3, 1), (80, 80, 5, 5), (256, 256, 2, 1), (6, 2, 3, 2),
                                               (10, 10, 1, 1), (96, 24, 7, 1), (1024, 1024, 1, 1), (128, 64, 40, 0), (34, 18, 2, 2)])
def test_layouts_and_sizes(ctx, dtype, interleaved, dim, rotated, hq, hk):
    rng = np.random.default_rng(dim + rotated + hq)
    past, new = [0, 7, 100000, 3], [1, 0, 40, 17]
    starts, lens = [0] + list(np.cumsum(new)), [p + n for p, n in zip(past, new)]
    pos = np.concatenate([np.arange(p, p + n) for p, n in zip(past, new)])
    table, freq = _table(rotated, interleaved, 1.0)
    parts = [_rows(58, h, dim, dtype, rng) for h in (hq, hk) if h]
    for inverse in (False, True):
        for place in ("in place", "out"):
            xs = [x.clone() for x, _ in parts]
            out = None if place == "in place" else tuple(torch.full_like(x, 9.0) for x in xs)
            got = ctx.rotary(table, *xs, starts=_ints(starts), lens=_ints(lens), max_new=40, inverse=inverse, out=out)
            ctx.sync()
            for (x, host), y, now in zip(parts, got, xs):
                _close(y, host, pos, freq, interleaved, 1.0, inverse, dtype)
                if place == "out":
                    assert torch.equal(now, x)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_and_negative_positions_and_a_factor(ctx, interleaved):
    rng = np.random.default_rng(2)
    pos = np.concatenate([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, 123456789], rng.integers(-2 ** 31, 2 ** 31, 50), rng.integers(0, 10 ** 6, 50)])
    freq = np.concatenate([[1.0, 0.0, 3.0, np.pi / 2], 10.0 ** -rng.uniform(0, 7, 28)]).astype(np.float32)
    table, freq = _table(64, interleaved, 1.37, freq=freq)
    q, host = _rows(len(pos), 3, 72, torch.float32, rng)
    got, none = ctx.rotary(table, q, positions=_ints(pos))
    ctx.sync()
    assert none is None and got is q
    _close(got, host, pos, freq, interleaved, 1.37, False, torch.float32)


@pytest.mark.parametrize("requests", [1, 255, 256, 257, 3000, 65535])
def test_many_requests(ctx, requests):
    """Rows are found among any number of requests, many of them empty."""
    rng = np.random.default_rng(requests)
    new = np.where(rng.random(requests) < 0.7, 0, rng.integers(0, 4, requests))
    new[-1] = 2
    lens, starts = new + rng.integers(0, 5000, requests), np.concatenate([[0], np.cumsum(new)])
    T = int(starts[-1])
    pos = np.repeat(lens - new, new) + np.arange(T) - np.repeat(starts[:-1], new)
    table, freq = _table(16, False)
    q, host = _rows(T + 5, 1, 16, torch.float32, rng)
    got, _ = ctx.rotary(table, q.clone(), starts=_ints(starts), lens=_ints(lens), max_new=int(new.max()))
    ctx.sync()
    _close(got[:T], host[:T], pos, freq, False, 1.0, False, torch.float32)
    assert torch.equal(got[T:], q[T:])                      # rows behind the last request's


def test_views_of_a_wider_matrix(ctx):
    """Queries and keys side by side with values, heads with room between them, and bases of any alignment."""
    rng = np.random.default_rng(3)
    table, freq = _table(32, False)
    for offset in (0, 1, 2, 4, 6):
        for dtype in (torch.bfloat16, torch.float32):
            buf = torch.from_numpy(rng.standard_normal((20, 7 * 64 + 16)).astype(np.float32)).to(dtype).to(DEV)
            before = buf.clone()
            q, k = buf[:, offset:offset + 256].view(20, 4, 64), buf[:, offset + 256:offset + 384].view(20, 2, 64)[:, :, :40]
            hosts = [t.double().cpu().numpy() for t in (q, k[..., :40])]
            ctx.rotary(table, q[..., :40], k, positions=_ints(np.arange(20)))
            ctx.sync()
            _close(q[..., :40], hosts[0][..., :40], np.arange(20), freq, False, 1.0, False, dtype)
            _close(k, hosts[1], np.arange(20), freq, False, 1.0, False, dtype)
            q[..., :40] = 0
            k[:] = 0
            before[:, offset:offset + 256].view(20, 4, 64)[..., :40] = 0
            before[:, offset + 256:offset + 384].view(20, 2, 64)[..., :40] = 0
            assert torch.equal(buf, before)


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_gradient(ctx, interleaved):
    """The inverse is the way back: against the formula's gradient, and the loss against its differences."""
    rng = np.random.default_rng(4)
    table, freq = _table(48, interleaved, 1.25)
    pos = rng.integers(0, 4000, 30)
    x, host = _rows(30, 3, 64, torch.float32, rng)
    dy, dhost = _rows(30, 3, 64, torch.float32, rng)
    got, _ = ctx.rotary(table, dy, positions=_ints(pos), inverse=True, out=torch.empty_like(dy))
    ctx.sync()
    _close(got, dhost, pos, freq, interleaved, 1.25, True, torch.float32)
    # sum of y dy is linear in x: its difference along any direction is that direction times the gradient
    step = rng.standard_normal(host.shape)
    diff = ((ref.rotary(host + step, pos, freq, interleaved, 1.25)[0] - ref.rotary(host - step, pos, freq, interleaved, 1.25)[0]) / 2 * dhost).sum()
    g = got.double().cpu().numpy()
    _, size = ref.rotary(dhost, pos, freq, interleaved, 1.25, True)
    assert abs(diff - (g * step).sum()) <= ((2.0 ** -24 * np.abs(g) + 2.0 ** -21 * size) * np.abs(step)).sum() + 1e-9


def test_requests_that_do_not_fit(ctx):
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SbError
    rng = np.random.default_rng(5)
    table, freq = _table(16, True)
    x, host = _rows(20, 2, 16, torch.bfloat16, rng)
    for case in range(4):
        starts, lens = [0, 4, 8, 20], [20, 40, 16]
        if case == 0: lens[2] = 11                            # fewer tokens than new ones
        if case == 1: starts[3] = 21                          # past the rows
        if case == 2: starts[3] = 7                           # backwards
        if case == 3: lens[2], starts[3] = 50, 20             # more than max_new
        got, _ = ctx.rotary(table, x.clone(), starts=_ints(starts), lens=_ints(lens), max_new=11 if case == 3 else 13)
        with pytest.raises(SbError) as e:
            ctx.sync()
        assert e.value.status == SB_ERR_INVALID
        _close(got[:8], host[:8], [16, 17, 18, 19, 36, 37, 38, 39], freq, True, 1.0, False, torch.bfloat16)
        assert torch.equal(got[8:], x[8:])
    none = x[:0]
    ctx.rotary(table, none, starts=_ints([0, 0]), lens=_ints([3]), max_new=0)
    ctx.rotary(table, none, positions=_ints(np.zeros(0)))
    ctx.sync()


def test_in_a_graph(ctx):
    """A captured step serves requests that grow."""
    from paper_2602_17698_b200.binding import Context
    rng = np.random.default_rng(6)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = Context(stream=side)
        table, freq = _table(64, False)
        q, host = _rows(3, 4, 64, torch.float32, rng)
        out, one, lens = torch.empty_like(q), _ints([0, 1, 2, 3]), _ints([5, 1, 700])
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.rotary(table, q, starts=one, lens=lens, max_new=1, out=out)
        for i in range(3):
            graph.replay()
            c.sync()
            _close(out, host, np.array([4, 0, 699]) + i, freq, False, 1.0, False, torch.float32)
            lens += 1
        del graph
        c.close()


def test_refusals(ctx):
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SB_ERR_SHAPE, RotaryTable, SbError
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    table, _ = _table(64, False)
    wide, _ = _table(66, False)
    pos = _ints([0, 1, 2, 3])
    back = RotaryTable(table.freq, factor=float("inf"))
    other = torch.zeros_like(x)
    alias = torch.zeros(4 * 2 * 128, dtype=torch.bfloat16, device=DEV)
    for status, call in [(SB_ERR_SHAPE, lambda: ctx.rotary(wide, x, positions=pos)), (SB_ERR_INVALID, lambda: ctx.rotary(back, x, positions=pos)),
                         (SB_ERR_SHAPE, lambda: ctx.rotary(table, torch.zeros(4, 1, 65, dtype=torch.bfloat16, device=DEV), positions=pos)),
                         (SB_ERR_SHAPE, lambda: ctx.rotary(table, torch.zeros(4, 1, 1026, dtype=torch.bfloat16, device=DEV), positions=pos)),
                         (SB_ERR_INVALID, lambda: ctx.rotary(table, x, starts=_ints([0, 4]), lens=_ints([4]), max_new=-1)),
                         (SB_ERR_SHAPE, lambda: ctx.rotary(table, alias[:512].view(4, 2, 64), positions=pos, out=alias.view(4, 4, 64)[:, ::2])),
                         # outputs on one another, on the other part, on themselves
                         (SB_ERR_INVALID, lambda: ctx.rotary(table, x, x, positions=pos)), (SB_ERR_INVALID, lambda: ctx.rotary(table, x, other, positions=pos, out=(other, x))),
                         (SB_ERR_INVALID, lambda: ctx.rotary(table, x, other, positions=pos, out=(alias[:512].view(4, 2, 64), alias[:512].view(4, 2, 64)))),
                         (SB_ERR_INVALID, lambda: ctx.rotary(table, x, other, positions=pos, out=(alias[:512].view(4, 2, 64), x))),
                         (SB_ERR_SHAPE, lambda: ctx.rotary(table, x[:, :1].expand(4, 2, 64), positions=pos)),
                         (SB_ERR_SHAPE, lambda: ctx.rotary(table, x, positions=pos, out=other[:1].expand(4, 2, 64)))]:
        with pytest.raises(SbError) as e:
            call()
        assert e.value.status == status
    for error, call in [(ValueError, lambda: ctx.rotary(table, x)), (ValueError, lambda: ctx.rotary(table, x, positions=pos[:3])),
                        (ValueError, lambda: ctx.rotary(table, x, positions=pos, starts=pos)), (TypeError, lambda: ctx.rotary(table, x.half(), positions=pos)),
                        (ValueError, lambda: ctx.rotary(table, x, x.float(), positions=pos)), (ValueError, lambda: ctx.rotary(table, x, x[:3], positions=pos)),
                        (ValueError, lambda: ctx.rotary(table, x[..., ::2], positions=pos)), (ValueError, lambda: ctx.rotary(table, x, x, positions=pos, out=x)),
                        (ValueError, lambda: ctx.rotary(table, x.cpu(), positions=pos))]:
        with pytest.raises(error):
            call()
    ctx.sync()
