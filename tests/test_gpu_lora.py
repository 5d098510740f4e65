"""Low-rank adapters of many requests against 64 bits."""
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


def _device(x, dtype=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(dtype).to(DEV)


class Case:
    def __init__(self, new, ids, inner, outer, rank, adapters, dtype=torch.bfloat16, seed=0, scaled=True, behind=0):
        from paper_2602_17698_b200.binding import LoraAdapters
        rng = np.random.default_rng(seed + inner + outer + rank + sum(new))
        self.starts, self.ids, self.max_new, self.dtype = [0] + [int(v) for v in np.cumsum(new)], list(ids), max(new), dtype
        T = self.starts[-1] + behind
        self.x = low.bf16(rng.standard_normal((T, inner)) * np.exp(rng.standard_normal(inner)))
        self.a, self.b = low.bf16(rng.standard_normal((adapters, rank, inner))), low.bf16(rng.standard_normal((adapters, outer, rank)))
        self.scale = rng.uniform(-2, 2, adapters).astype(np.float32) if scaled else None
        self.base = _device(rng.standard_normal((T, outer)) * 10, dtype)
        self.adapters = LoraAdapters(_device(self.a), _device(self.b), None if self.scale is None else _device(self.scale, torch.float32))
        self.args = (_ints(self.ids), _ints(self.starts), self.max_new)

    def check(self, got, rows=None):
        """All rows, or those of a slice."""
        T = self.starts[-1]
        base = self.base.double().cpu().numpy()
        want, second, first = ref.lora(self.x, base, self.a, self.b, self.scale, self.ids, self.starts)
        inner, rank = self.a.shape[2], self.a.shape[1]
        # the result's rounding; sums in fp32 by the tensor cores, which may cut off a unit, 2^-23, at each step of 16 and where parts are
        # added, of the magnitudes; what two bf16 numbers leave of the inner sums, 2^-17; the scale
        tol = HALF_STEP[self.dtype] * np.abs(want) + 2.0 ** -23 * ((inner / 16 + 40) * first + (rank / 8 + 4) * second) + 2.0 ** -17 * second \
            + 2.0 ** -23 * np.abs(base)
        err = np.abs(got.double().cpu().numpy() - want)
        err, tol = (t[:T][slice(None) if rows is None else rows] for t in (err, tol))
        assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err - tol).argmax(), err.shape))
        return T


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new,ids,inner,outer,rank,adapters", [
    ([1], [0], 8, 1, 8, 1), ([1], [2], 4096, 512, 16, 3), ([1] * 20, list(range(20)), 256, 96, 8, 20), ([1, 0, 3, 5], [1, 0, -1, 1], 520, 264, 24, 2),
    ([16, 15, 1], [0, 1, 0], 1000, 333, 32, 2), ([17], [0], 64, 40, 64, 1), ([100, 0, 1, 64], [1, 1, 0, -1], 776, 100, 40, 2),
    ([65, 63], [0, 0], 2048, 1032, 128, 1), ([200, 33], [1, 0], 136, 77, 104, 2), ([130], [0], 4104, 256, 16, 1), ([300, 5, 70], [2, 1, 0], 512, 640, 64, 3),
    ([90], [-1], 64, 50, 8, 1), ([90, 80], [1, 0], 1032, 200, 24, 2), ([80], [0], 6000, 300, 32, 1), ([1], [0], 14336, 4100, 128, 1), ([3], [0], 9000, 9000, 64, 1),
    ([20] * 40, [i % 7 - 1 for i in range(40)], 1024, 128, 32, 6), ([2, 16], [1, 1], 14336, 64, 48, 2)])
def test_sizes(ctx, dtype, new, ids, inner, outer, rank, adapters):
    case = Case(new, ids, inner, outer, rank, adapters, dtype)
    x, base = _device(case.x), case.base.clone()
    out = torch.full_like(base, 9.0)
    assert ctx.lora_add(case.adapters, x, base, *case.args, out=out) is out
    ctx.sync()
    case.check(out)
    assert torch.equal(base, case.base)
    got = ctx.lora_add(case.adapters, x, base, *case.args)          # in place
    ctx.sync()
    assert got is base and torch.equal(got, out)


@pytest.mark.parametrize("new", [[1, 2], [70, 20]])
def test_no_scale_and_rows_behind_the_last(ctx, new):
    case = Case(new, [0, 1], 256, 128, 16, 2, scaled=False, behind=9)
    out = torch.full_like(case.base, 9.0)
    ctx.lora_add(case.adapters, _device(case.x), case.base, *case.args, out=out)
    ctx.sync()
    T = case.check(out)
    assert (out[T:] == 9).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [[3, 2], [70, 20]])
@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 3), (2, 2), (4, 0), (8, 24)])
def test_views_of_wider_matrices(ctx, dtype, new, offset, pad):
    """Rows of any pitch and alignment; what lies beside them stays."""
    case = Case(new, [0, 1], 264, 70, 16, 2, dtype)
    T = case.starts[-1]
    xbuf = torch.zeros(T, 264 + 16, dtype=torch.bfloat16, device=DEV)
    xbuf[:, 8:272] = _device(case.x)
    buf = torch.full((T, 70 + offset + pad), 5.0, dtype=dtype, device=DEV)
    y = buf[:, offset:offset + 70]
    y.copy_(case.base)
    ctx.lora_add(case.adapters, xbuf[:, 8:272], y, *case.args)
    ctx.sync()
    case.check(y)
    y.fill_(5.0)
    assert (buf == 5).all()


@pytest.mark.parametrize("requests", [255, 256, 257, 2000])
def test_many_requests(ctx, requests):
    rng = np.random.default_rng(requests)
    new = np.where(rng.random(requests) < 0.8, 0, rng.integers(0, 30, requests))
    new[-1] = 40
    case = Case(list(new), rng.integers(-1, 5, requests), 64, 48, 8, 5)
    out = torch.empty_like(case.base)
    ctx.lora_add(case.adapters, _device(case.x), case.base, *case.args, out=out)
    ctx.sync()
    case.check(out)


def test_infinities_stay_where_they_are(ctx):
    """What is not finite in one row, or in an adapter that no row has, reaches no other row."""
    for new in ([2, 3], [40, 30]):
        case = Case(new, [0, 2], 128, 64, 16, 3)
        x = _device(case.x)
        case.adapters.a[1], case.adapters.b[1] = float("nan"), float("inf")
        x[1] = float("nan")
        x[0, 3] = float("inf")
        out = ctx.lora_add(case.adapters, x, case.base, *case.args, out=torch.empty_like(case.base))
        ctx.sync()
        # (an infinity meets weights of both signs: inf - inf)
        assert not torch.isfinite(out[:2].float()).any() and torch.isnan(out[1].float()).all()
        case.x[:2] = 0
        case.check(out, slice(2, None))


@pytest.mark.parametrize("new", [[2], [40]])
def test_an_infinity_stays_one(ctx, new):
    case = Case(new, [0], 128, 64, 16, 1, scaled=False)
    case.adapters.a.abs_()
    case.adapters.b.abs_()
    x = _device(case.x)
    x[1, 5] = float("inf")
    out = ctx.lora_add(case.adapters, x, case.base, *case.args, out=torch.empty_like(case.base))
    ctx.sync()
    assert (out[1] == float("inf")).all() and torch.isfinite(out[[i for i in range(len(out)) if i != 1]].float()).all()


def test_requests_and_ids_that_do_not_fit(ctx):
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SbError
    for rows in (4, 30):
        for bad in range(6):
            case = Case([rows, rows, rows], [0, 1, 0], 64, 40, 8, 2)
            starts, ids = list(case.starts), list(case.ids)
            if bad == 0: starts[3] = 3 * rows + 1                 # past the rows
            if bad == 1: starts[3] = 2 * rows - 1                 # backwards
            if bad == 2: ids[2] = 2                               # no such adapter
            if bad == 3: ids[2] = -2
            if bad == 4: starts[0] = -1
            if bad == 5: starts[2] = rows - 1                     # one backwards, one too long
            out = torch.full_like(case.base, 9.0)
            ctx.lora_add(case.adapters, _device(case.x), case.base, _ints(ids), _ints(starts), rows, out=out)
            with pytest.raises(SbError) as e:
                ctx.sync()
            assert e.value.status == SB_ERR_INVALID
            first, second, third = (slice(i * rows, (i + 1) * rows) for i in range(3))
            served = {0: (first, second), 1: (first, second), 2: (first, second), 3: (first, second), 4: (second, third), 5: (first,)}[bad]
            left = {0: (third,), 1: (third,), 2: (), 3: (), 4: (first,), 5: (second, third)}[bad]
            for s in served:
                case.check(out, s)
            for s in left:
                assert (out[s] == 9).all()
            if bad in (2, 3):                                       # counts as having none
                assert torch.equal(out[third], case.base[third])


@pytest.mark.parametrize("new", [1, 40])
def test_same_sums_every_time_and_in_a_graph(ctx, new):
    """A captured step serves requests whose adapters change."""
    from paper_2602_17698_b200.binding import Context
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = Context(stream=side)
        case = Case([new] * 12, [i % 5 for i in range(12)], 4096, 256, 16, 5)
        x, out = _device(case.x), torch.empty_like(case.base)
        ids, starts, n = case.args
        c.lora_add(case.adapters, x, case.base, ids, starts, n, out=out)
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.lora_add(case.adapters, x, case.base, ids, starts, n, out=out)
        for i in range(6):
            case.ids = [(j + i) % 6 - 1 for j in range(12)]
            ids.copy_(_ints(case.ids))
            graph.replay()
            again = c.lora_add(case.adapters, x, case.base, ids, starts, n, out=torch.empty_like(out))
            c.sync()
            case.check(out)
            assert torch.equal(out, again)
        del graph
        c.close()


def test_two_contexts_at_once():
    """Each with its own stream and scratch; the sums are those of a call alone."""
    from paper_2602_17698_b200.binding import Context
    runs = []
    for new in ([90, 5, 70], [3, 1, 2], [400, 0, 33]):
        case = Case(new, [1, 0, 1], 2048, 1000, 64, 2)
        runs.append((case, Context(stream=torch.cuda.Stream()), _device(case.x), [torch.empty_like(case.base) for _ in range(6)]))
    torch.cuda.synchronize()
    for i in range(6):
        for case, c, x, outs in runs:
            c.lora_add(case.adapters, x, case.base, *case.args, out=outs[i])
    for case, c, x, outs in runs:
        c.sync()
        case.check(outs[0])
        assert all(torch.equal(o, outs[0]) for o in outs)
        c.close()


def test_nothing_to_do_and_refusals(ctx):
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SB_ERR_SHAPE, LoraAdapters, SbError, lib
    case = Case([2, 1], [0, 1], 64, 40, 8, 2)
    x, (ids, starts, n) = _device(case.x), case.args
    ctx.lora_add(case.adapters, x[:0], case.base[:0], ids, torch.zeros_like(starts), 0)

    def direct(adapters=case.adapters.struct, ldx=64, ldb=40, ldy=40, y=None, f32=0, xp=x.data_ptr(), max_new=2):
        return lambda: ctx._check(lib().sb_lora_add(ctx._h, adapters, xp, ldx, case.base.data_ptr(), ldb, y or case.base.data_ptr(), ldy, f32, 3,
                                                    starts.data_ptr(), ids.data_ptr(), 2, max_new))
    calls = [(SB_ERR_SHAPE, direct(ldx=60)), (SB_ERR_SHAPE, direct(ldx=68)), (SB_ERR_SHAPE, direct(xp=x.data_ptr() + 2)), (SB_ERR_SHAPE, direct(ldb=39)),
             (SB_ERR_SHAPE, direct(ldy=41)), (SB_ERR_SHAPE, direct(y=case.base.data_ptr() + 1)), (SB_ERR_INVALID, direct(f32=2)),
             (SB_ERR_INVALID, direct(max_new=-1)), (SB_ERR_INVALID, direct(y=x.data_ptr()))]
    for field, value, status in (("rank", 4, SB_ERR_SHAPE), ("rank", 136, SB_ERR_SHAPE), ("in_", 60, SB_ERR_SHAPE), ("adapters", 0, SB_ERR_INVALID),
                                 ("a", None, SB_ERR_INVALID), ("b", case.adapters.b.data_ptr() + 8, SB_ERR_SHAPE), ("out", 0, SB_ERR_INVALID)):
        ad = LoraAdapters(case.adapters.a, case.adapters.b)
        setattr(ad.struct, field, value)
        calls.append((status, direct(ad.struct)))
    for status, call in calls:
        with pytest.raises(SbError) as e:
            call()
        assert e.value.status == status
    for error, call in [(ValueError, lambda: ctx.lora_add(case.adapters, x[:, :56], case.base, ids, starts, n)),
                        (ValueError, lambda: ctx.lora_add(case.adapters, x, case.base[:, :39], ids, starts, n)),
                        (TypeError, lambda: ctx.lora_add(case.adapters, x, case.base.half(), ids, starts, n)),
                        (TypeError, lambda: ctx.lora_add(case.adapters, x, case.base, ids, starts, n, out=case.base.float())),
                        (ValueError, lambda: ctx.lora_add(case.adapters, x, case.base, ids[:1], starts, n)),
                        (ValueError, lambda: ctx.lora_add(case.adapters, x, case.base, ids.long(), starts, n)),
                        (TypeError, lambda: LoraAdapters(case.adapters.a.float(), case.adapters.b)),
                        (ValueError, lambda: LoraAdapters(case.adapters.a, case.adapters.b[:, :, :4].contiguous()))]:
        with pytest.raises(error):
            call()
    ctx.sync()
