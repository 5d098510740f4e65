"""The 4-bit key/value cache: appending bit for bit, attention against 64 bits."""
import numpy as np
import pytest
import torch

import lowbit_reference as low
import more_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    c = Context()
    yield c
    c.close()


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def _starts(n):
    return [0] + list(np.cumsum(n))


def _cache(lens, heads, page, dim, rng, spare=3, head_scales=True):
    per = max(1, max(-(-ln // page) for ln in lens))
    table = rng.permutation(per * len(lens) + spare)[:per * len(lens)].reshape(len(lens), per).astype(np.int64)
    return ref.Cache4(per * len(lens) + spare, heads, page, dim, table, rng, head_scales)


def _same(cache, dev):
    for side, (code, scale) in enumerate(((dev.k, dev.k_scale), (dev.v, dev.v_scale))):
        q, s = cache.bytes(side)
        np.testing.assert_array_equal(scale.cpu().numpy(), s)
        np.testing.assert_array_equal(code.cpu().numpy(), q)


def _tokens(T, heads, dim, rng, spread=1.0):
    return low.bf16(rng.standard_normal((T, heads, dim)) * np.exp(spread * rng.standard_normal((T, 1, 1))))


def _device(x):
    return torch.from_numpy(x).to(torch.bfloat16).to(DEV)


# ---- appending --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("past,new,heads,page,dim", [
    ([0], [1], 1, 16, 16), ([15], [1], 2, 16, 128), ([16], [1], 2, 16, 128), ([7, 0, 33], [1, 1, 1], 8, 64, 128), ([5, 9], [3, 2], 3, 16, 48),
    ([5, 40, 0, 100], [70, 0, 33, 1], 3, 48, 80), ([0, 3], [500, 16], 2, 32, 64), ([31, 1], [2, 40], 1, 128, 256), ([1], [300], 4, 16, 96),
    ([2, 70], [11, 5], 5, 16, 208)])
@pytest.mark.parametrize("head_scales", [True, False])
def test_append_is_exact(ctx, past, new, heads, page, dim, head_scales):
    rng = np.random.default_rng(sum(past) + 3 * sum(new) + dim)
    lens, starts = [p + n for p, n in zip(past, new)], _starts(new)
    cache = _cache(lens, heads, page, dim, rng, head_scales=head_scales)
    dev = cache.device(DEV)
    k, v = _tokens(starts[-1], heads, dim, rng), _tokens(starts[-1], heads, dim, rng)
    for side, x in enumerate((k, v)):
        cache.append(side, x, starts, lens)
    for _ in range(2):                         # the second time changes nothing
        ctx.kv4_append(dev, _device(k), _device(v), _ints(starts), _ints(lens), max(new))
        ctx.sync()
        _same(cache, dev)
    gk, gv = ctx.kv4_read(dev, _ints(starts), _ints(lens), max(new))
    ctx.sync()
    for side, x in enumerate((gk, gv)):
        want = np.concatenate([cache.values(side, b, ln)[:, p:].transpose(1, 0, 2) for b, (p, ln) in enumerate(zip(past, lens))])
        np.testing.assert_array_equal(x.float().cpu().numpy(), low.bf16(want))


@pytest.mark.parametrize("g", [1.0, 2.0 ** -40, 3e20, 1e-30])
def test_zeros_and_extreme_sizes(ctx, g):
    rng = np.random.default_rng(4)
    new, heads, dim = 80, 2, 128
    cache = _cache([new], heads, 16, dim, rng)
    cache.head = [np.full(heads, g, np.float32), np.array([g, 1], np.float32)]
    dev = cache.device(DEV)
    x = low.bf16(rng.standard_normal((new, heads, dim)))
    x[:16] = 0
    x[16:32] *= np.float32(2.0) ** -132                        # subnormal numbers
    x[32:48] = low.bf16(x[32:48] * np.float32(2.0 ** 124))
    x[48:64, 0] = 0
    x[64:70] *= np.float32(g)
    x = low.bf16(x)
    for side in range(2):
        cache.append(side, x, [0, new], [new])
    ctx.kv4_append(dev, _device(x), _device(x), _ints([0, new]), _ints([new]), new)
    ctx.sync()
    _same(cache, dev)


def test_ties_and_the_ends_of_the_scale(ctx):
    """Every bf16 number of two binades over a block whose largest element is 6, so the scale is 1: each code's border is among them."""
    rng = np.random.default_rng(5)
    cache = _cache([32], 1, 16, 256, rng, head_scales=False)
    dev = cache.device(DEV)
    x = (np.arange(32 * 256, dtype=np.uint32) << 16).view(np.float32)[None].copy()
    bits = (np.linspace(0x3e00, 0x40c0, 32 * 240).astype(np.uint32) << 16)
    x = np.zeros((32, 1, 16, 16), np.float32)
    x[..., 1:] = bits.view(np.float32).reshape(32, 1, 16, 15) * np.where(rng.random((32, 1, 16, 15)) < 0.5, -1, 1)
    x[..., 0] = 6
    x = x.reshape(32, 1, 256)
    for side in range(2):
        cache.append(side, x, [0, 32], [32])
    ctx.kv4_append(dev, _device(x), _device(x), _ints([0, 32]), _ints([32]), 32)
    ctx.sync()
    _same(cache, dev)


def test_not_a_number_is_stored_as_zero_and_reported(ctx):
    from paper_2602_17698_b200.binding import SB_ERR_NONFINITE, SbError
    rng = np.random.default_rng(4)
    for bad in ("elements", "head scale"):
        cache = _cache([40], 3, 16, 64, rng)
        x = _tokens(40, 3, 64, rng, 0)
        if bad == "elements":
            x[3, 0, 5], x[20, 0, 6], x[20, 0, 7], x[30, 2] = np.nan, np.inf, -np.inf, np.nan
        else:
            cache.head[0][:] = [np.nan, 0, -1]
            cache.head[1][:] = [np.inf, 1, 2]
        dev = cache.device(DEV)
        ctx.kv4_append(dev, _device(x), _device(x), _ints([0, 40]), _ints([40]), 40)
        with pytest.raises(SbError) as e:
            ctx.sync()
        assert e.value.status == SB_ERR_NONFINITE
        for side in range(2):
            cache.append(side, x, [0, 40], [40])
        _same(cache, dev)
        ctx.sync()


def test_rows_of_a_wider_matrix(ctx):
    rng = np.random.default_rng(9)
    cache = _cache([40, 40], 2, 32, 64, rng)
    dev = cache.device(DEV)
    for step in range(20):
        lens, starts = [step + 1, step + 7], _starts([1, 1])
        qkv = low.bf16(rng.standard_normal((2, 6 * 64)))
        k, v = (qkv[:, i * 128:(i + 1) * 128].reshape(2, 2, 64) for i in (1, 2))
        d = _device(qkv)
        ctx.kv4_append(dev, d[:, 128:256].view(2, 2, 64), d[:, 256:].view(2, 2, 64), _ints(starts), _ints(lens), 1)
        for side, x in enumerate((k, v)):
            cache.append(side, x, starts, lens)
    ctx.sync()
    _same(cache, dev)


def test_requests_that_do_not_fit_are_skipped_and_reported(ctx):
    """Numbers on the device that do not fit: nothing is read or written outside, the others are served."""
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SbError
    rng = np.random.default_rng(8)
    heads, dim, page = 2, 64, 16
    for rows in (4, 12, 30):
        held = [20, 40, 16] if rows < 16 else [60, 80, 48]
        cache = _cache(held, heads, page, dim, rng, spare=0)
        x, q = _tokens(5 * rows, heads, dim, rng), _tokens(5 * rows, 2 * heads, dim, rng)
        for case in range(6):
            dev = cache.device(DEV)
            lens, starts = list(held), [0, rows, 2 * rows, 3 * rows]
            if case == 0: lens[2] = 1000                          # more tokens than pages
            if case == 1: lens[2] = 3                             # fewer tokens than new ones
            if case == 2: starts[3] = 5 * rows + 1                # past the dense rows
            if case == 3: starts[3] = 2 * rows - 1                # backwards
            if case == 4: dev.table[2] = 10 ** 6                  # no such page
            if case == 5: dev.table[2] = -1
            before = [t.clone() for t in (dev.k, dev.v)]
            for call in ("append", "read", "attention"):
                out = torch.full((5 * rows, 2 * heads, dim), 7.0, dtype=torch.bfloat16, device=DEV)
                if call == "append":
                    ctx.kv4_append(dev, _device(x), _device(x), _ints(starts), _ints(lens), rows)
                elif call == "read":
                    got = [out[:, :heads].contiguous(), out[:, heads:].contiguous()]
                    ctx.kv4_read(dev, _ints(starts), _ints(lens), rows, out=got)
                    out = torch.cat(got, 1)
                else:
                    ctx.kv4_attention(dev, _device(q), _ints(starts), _ints(lens), rows, 96, out=out)
                with pytest.raises(SbError) as e:
                    ctx.sync()
                assert e.value.status == SB_ERR_INVALID
                if call == "append":
                    for t, b in zip((dev.k, dev.v), before):
                        assert torch.equal(t[cache.table[2]], b[cache.table[2]]) and not torch.equal(t, b)
                else:
                    assert (out[:2 * rows] != 7).any() and torch.isfinite(out.float()).all()


# ---- attention --------------------------------------------------------------------------------------------------

def _attend(ctx, past, new, heads, group, page, dim, window=0, scale=None, qsize=1.0, max_len=None, seed=0, poison=True, wide=False, change=None,
            head_scales=True):
    rng = np.random.default_rng(seed + sum(past) + 3 * sum(new) + dim + 11 * group)
    lens, starts = [p + n for p, n in zip(past, new)], _starts(new)
    cache = _cache(lens, heads, page, dim, rng, head_scales=head_scales)
    if change:
        change(cache)
    dev = cache.device(DEV)
    if poison:
        # slots past a request's end hold anything: NaN scales
        for b, ln in enumerate(lens):
            for p in range(ln, cache.table.shape[1] * page):
                pg, slot = int(cache.table[b, p // page]), p % page
                dev.k[pg, :, slot] = 0x7f
                dev.v[pg, :, slot] = 0xff
                dev.k_scale[pg, :, slot] = 0x7f
                dev.v_scale[pg, :, slot] = 0xff
    T = starts[-1]
    q = low.bf16(rng.standard_normal((T, heads * group, dim)) * qsize)
    qd, out = _device(q), None
    if wide:
        buf = torch.zeros(T, heads * group * dim + 64, dtype=torch.bfloat16, device=DEV)
        buf[:, :-64] = qd.view(T, -1)
        qd = buf[:, :-64].view(T, heads * group, dim)
        obuf = torch.full((T, heads * group + 2, dim + 8), 5.0, dtype=torch.bfloat16, device=DEV)
        out = obuf[:, :-2, :-8]
    sc = dim ** -0.5 if scale is None else scale
    out, lse = ctx.kv4_attention(dev, qd, _ints(starts), _ints(lens), max(new), max(lens) if max_len is None else max_len, scale=scale,
                                 window=window, out=out, want_lse=True)
    ctx.sync()
    want, wlse, mag, top, held = ref.attention(cache, q, starts, lens, sc, window)
    # the last rounding, 2^-8 of the result; every weight rounded to fp16, 2^-11 of weight x |v|, and where it falls below fp16's normal
    # numbers an absolute 2^-25, where the row's largest is 2^6 at least; scores summed in fp32, 2^-20 of their terms' magnitudes,
    # which moves a weight by that much
    eps = 2.0 ** -20 * (top + 1)
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * eps[..., None]) * mag + 2.0 ** -31 * held + 1e-30
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
    lerr = np.abs(lse.double().cpu().numpy() - wlse)
    assert (lerr <= eps + 2.0 ** -21 * np.abs(wlse)).all(), float((lerr / eps).max())
    if wide:
        assert (obuf[:, -2:] == 5).all() and (obuf[:, :, -8:] == 5).all()


@pytest.mark.parametrize("past,new,heads,group,page,dim", [
    ([0], [1], 1, 1, 16, 128), ([1], [1], 2, 4, 16, 64), ([15, 16, 17], [1, 1, 1], 2, 8, 16, 128), ([100, 0, 63], [1, 0, 1], 1, 5, 48, 80),
    ([500, 31, 32, 33], [1, 1, 1, 1], 4, 4, 64, 128), ([700], [1], 1, 12, 32, 256), ([90, 200], [1, 1], 2, 3, 128, 16), ([77], [1], 2, 2, 16, 48),
    ([130], [1], 1, 4, 16, 144), ([130, 7], [1, 1], 1, 4, 16, 208), ([66], [1], 2, 20, 16, 96)])
def test_one_token_per_request(ctx, past, new, heads, group, page, dim):
    _attend(ctx, past, new, heads, group, page, dim)


@pytest.mark.parametrize("past,new,heads,group,page,dim", [
    ([40, 3], [5, 2], 2, 4, 16, 128), ([0], [33], 1, 2, 16, 64), ([17, 0, 64], [40, 70, 0], 2, 3, 32, 128), ([30], [20], 1, 7, 48, 256),
    ([0, 100], [130, 1], 1, 4, 64, 96), ([5], [150], 1, 8, 16, 128), ([0, 257], [300, 129], 2, 1, 64, 128), ([9], [60], 1, 3, 16, 16),
    ([9, 50], [60, 33], 1, 3, 16, 48), ([9], [60], 1, 3, 16, 112), ([9], [60], 1, 3, 16, 144),
    ([0, 33], [130, 1], 1, 2, 64, 208)])
def test_drafts_and_prompts(ctx, past, new, heads, group, page, dim):
    _attend(ctx, past, new, heads, group, page, dim)


@pytest.mark.parametrize("window", [1, 2, 16, 50, 129])
@pytest.mark.parametrize("past,new", [([200, 10], [1, 1]), ([300, 0], [6, 9]), ([150, 0], [40, 140])])
def test_sliding_window(ctx, window, past, new):
    _attend(ctx, past, new, 2, 4, 32, 64, window=window)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_long_cache_in_many_chunks(ctx, dim):
    _attend(ctx, [9000, 1234], [1, 3], 1, 4, 64, dim, poison=False)


@pytest.mark.parametrize("past,new,heads,group,dim,window", [
    ([3000], [70], 1, 4, 128, 0), ([2500, 10], [33, 65], 2, 3, 64, 0), ([1500], [257], 1, 1, 96, 0), ([4000, 0], [40, 64], 1, 4, 80, 700),
    ([0], [129], 1, 2, 128, 0), ([1111, 0, 127], [20, 0, 40], 2, 5, 128, 0),
    ([1900, 40], [50, 90], 2, 4, 256, 0), ([700], [64], 1, 4, 240, 300), ([0, 1000], [128, 129], 1, 1, 256, 0)])
def test_chunks_of_prompts_behind_a_long_past(ctx, past, new, heads, group, dim, window):
    _attend(ctx, past, new, heads, group, 16, dim, window=window)


@pytest.mark.parametrize("past,new", [([2900, 40], [30, 20]), ([2900, 40], [2, 1])])
@pytest.mark.parametrize("max_len", [1, 100, 1500, 10 ** 6])
def test_max_len_decides_nothing_but_the_chunks(ctx, max_len, past, new):
    _attend(ctx, past, new, 1, 4, 32, 128, max_len=max_len, poison=False)


def test_strided_queries_and_outputs(ctx):
    _attend(ctx, [70, 20], [3, 40], 2, 2, 16, 128, wide=True)
    _attend(ctx, [70, 20], [3, 1], 2, 2, 16, 128, wide=True)


@pytest.mark.parametrize("qsize", [1e-30, 1e-4, 30.0, 1e4])
@pytest.mark.parametrize("new", [[1, 2], [1, 30]])
def test_sizes_of_queries(ctx, qsize, new):
    """From scores that are all equal to ones that pick a single key; fp16 alone would lose both ends."""
    _attend(ctx, [300, 40], new, 1, 4, 16, 64, qsize=qsize, scale=0.125 if qsize < 1e3 else 1e-5)


@pytest.mark.parametrize("scale", [-0.1, 0.0, -3.0])
@pytest.mark.parametrize("new", [[1, 2], [40, 5]])
def test_scales_of_the_softmax(ctx, scale, new):
    _attend(ctx, [300, 40], new, 1, 4, 16, 128, scale=scale)


@pytest.mark.parametrize("new", [[1, 2], [40, 5]])
def test_scales_of_very_different_sizes(ctx, new):
    def change(cache):
        for side in range(2):
            cache.scale[side] = low.round_e4m3(np.exp2(np.random.default_rng(side).uniform(-11, 9, cache.scale[side].shape))).astype(np.float32)
        cache.head[0][:] = 2.0 ** -7
        cache.head[1][:] = 1e5
        cache.scale[1][cache.table[0, 1]] = 0
        cache.scale[0][cache.table[0, 2]] = 0
    _attend(ctx, [400, 60], new, 1, 4, 16, 128, change=change)


@pytest.mark.parametrize("new", [[2], [40]])
def test_a_cache_of_zeros_and_heads_without_scales(ctx, new):
    def change(cache):
        cache.scale[1][:] = 0
    _attend(ctx, [100], new, 1, 2, 16, 128, change=change)
    _attend(ctx, [100], new, 2, 2, 16, 128, head_scales=False)


@pytest.mark.parametrize("new", [[2], [40]])
@pytest.mark.parametrize("up", [True, False])
def test_a_maximum_that_moves(ctx, new, up):
    """Keys that grow (or shrink) along the cache: the running maximum moves often (or never again)."""
    def change(cache):
        p = np.arange(cache.table.shape[1] * cache.page)
        size = np.exp2(np.linspace(-6, 6, len(p))[::1 if up else -1])
        page, slot = cache.table[0, p // cache.page], p % cache.page
        cache.scale[0][page, :, slot] = low.round_e4m3(size).astype(np.float32)[:, None, None]
    _attend(ctx, [1500], new, 1, 4, 16, 64, change=change, qsize=2.0)


def test_offsets_beyond_32_bits(ctx):
    """Pages near the end of a cache of more than 2^32 bytes give what the same pages at its start give."""
    from paper_2602_17698_b200.binding import Kv4Cache
    rng = np.random.default_rng(2)
    cache = _cache([300, 70], 1, 64, 128, rng, spare=0)
    small = cache.device(DEV)
    n, pages = cache.code[0].shape[0], (1 << 32) // (64 * 64) + 5000
    big = [torch.empty(pages, 1, 64, 64, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scale = [torch.empty(pages, 1, 64, 8, dtype=torch.uint8, device=DEV) for _ in range(2)]
    for t, s, code, sc in zip(big, scale, (small.k, small.v), (small.k_scale, small.v_scale)):
        t[-n:], s[-n:] = code, sc
    far = Kv4Cache(big[0], big[1], scale[0], scale[1], small.table + (pages - n), 128, small.k_head, small.v_head)
    for new in ([1, 1], [3, 40]):
        starts, lens = _starts(new), [300, 70]
        x, q = _device(_tokens(sum(new), 1, 128, rng)), _device(_tokens(sum(new), 4, 128, rng))
        outs = []
        for c in (small, far):
            ctx.kv4_append(c, x, x, _ints(starts), _ints(lens), max(new))
            outs.append((*ctx.kv4_attention(c, q, _ints(starts), _ints(lens), max(new), 300, want_lse=True),
                         *ctx.kv4_read(c, _ints(starts), _ints(lens), max(new))))
        ctx.sync()
        for a, b in zip(*outs):
            assert torch.equal(a, b)
    del far, big, t
    torch.cuda.empty_cache()


def test_same_sums_every_time_and_in_a_graph(ctx):
    """A captured step serves requests that grow: lengths and tables are read on the device."""
    from paper_2602_17698_b200.binding import Context
    rng = np.random.default_rng(3)
    heads, group, dim, page = 2, 4, 128, 16
    cache = _cache([5000, 100, 64], heads, page, dim, rng)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = Context(stream=side)
        dev, again = cache.device(DEV), cache.device(DEV)
        one, lens = _ints([0, 1, 2, 3]), _ints([4000, 80, 1])
        x, q = _device(_tokens(3, heads, dim, rng)), _device(_tokens(3, heads * group, dim, rng))
        out, lse = torch.empty(3, heads * group, dim, dtype=torch.bfloat16, device=DEV), torch.empty(3, heads * group, device=DEV)

        def step(d, o=out, s=lse):
            c.kv4_append(d, x, x, one, lens, 1)
            c.kv4_attention(d, q, one, lens, 1, 5000, out=o, lse=s)
        step(dev)
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(dev)
        for i in range(20):
            x.copy_(_device(_tokens(3, heads, dim, rng)))
            q.copy_(_device(_tokens(3, heads * group, dim, rng)))
            graph.replay()
            o2, l2 = torch.empty_like(out), torch.empty_like(lse)
            step(again, o2, l2)
            c.sync()
            assert torch.equal(out, o2) and torch.equal(lse, l2)
            lens += 1
        del graph
        c.close()


def test_nothing_new_and_results_on_another_stream(ctx):
    """Calls with no rows do nothing; results that the binding allocates belong to the context's stream."""
    from paper_2602_17698_b200.binding import Context
    rng = np.random.default_rng(1)
    cache = _cache([90, 70], 2, 16, 64, rng)
    dev = cache.device(DEV)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_append(dev, none, none, _ints([0, 0, 0]), _ints([90, 70]), 0)
    ctx.kv4_attention(dev, none, _ints([0, 0, 0]), _ints([90, 70]), 0, 90)
    q = _device(_tokens(50, 8, 64, rng))
    starts, lens = _ints([0, 20, 50]), _ints([90, 70])
    want = [*ctx.kv4_attention(dev, q, starts, lens, 30, 90, want_lse=True), *ctx.kv4_read(dev, starts, lens, 30, total=50)]
    ctx.sync()
    _same(cache, dev)
    side = torch.cuda.Stream()
    c = Context(stream=side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = [*c.kv4_attention(dev, q, starts, lens, 30, 90, want_lse=True), *c.kv4_read(dev, starts, lens, 30, total=50)]
    mine = [torch.full_like(t, 7.0) for t in got]
    c.sync()
    for a, b, m in zip(got, want, mine):
        assert torch.equal(a, b) and (m == 7).all()
    c.close()


def test_refusals(ctx):
    """What the host can see is refused before anything is enqueued."""
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SB_ERR_SHAPE, SbError
    rng = np.random.default_rng(1)
    cache = _cache([90, 70], 2, 16, 64, rng)
    q, x = _device(_tokens(2, 8, 64, rng)), _device(_tokens(2, 2, 64, rng))
    starts, lens = _ints([0, 1, 2]), _ints([90, 70])
    odd = torch.zeros(2 * 4 * 64 + 8, dtype=torch.bfloat16, device=DEV)

    def attend(dev, q=q, **kw):
        args = dict(max_new=1, max_len=90)
        args.update(kw)
        return lambda: ctx.kv4_attention(dev, q, starts, lens, args.pop("max_new"), args.pop("max_len"), **args)
    good = cache.device(DEV)
    calls = [(SB_ERR_INVALID, attend(good, max_len=0)), (SB_ERR_INVALID, attend(good, window=-1)), (SB_ERR_INVALID, attend(good, scale=float("nan"))),
             (SB_ERR_INVALID, attend(good, max_new=-1)), (SB_ERR_SHAPE, attend(good, q=_device(_tokens(2, 3, 64, rng)))),
             (SB_ERR_SHAPE, attend(good, q=odd[1:513].view(2, 4, 64))),
             (SB_ERR_SHAPE, lambda: ctx.kv4_append(good, odd[1:257].view(2, 2, 64), x, starts, lens, 1))]
    both = torch.empty_like(x)
    calls.append((SB_ERR_INVALID, lambda: ctx.kv4_read(good, starts, lens, 1, out=(both, both))))
    for field, value, status in (("page_tokens", 24, SB_ERR_SHAPE), ("dim", 72, SB_ERR_SHAPE), ("dim", 272, SB_ERR_SHAPE), ("heads", 0, SB_ERR_INVALID),
                                 ("pages", 0, SB_ERR_INVALID), ("table", None, SB_ERR_INVALID), ("k", good.k.data_ptr() + 8, SB_ERR_SHAPE),
                                 ("v_scale", good.v_scale.data_ptr() + 4, SB_ERR_SHAPE), ("requests", 70000, SB_ERR_SHAPE),
                                 ("table_stride", -1, SB_ERR_INVALID), ("table_pages", -1, SB_ERR_INVALID)):
        from paper_2602_17698_b200.binding import lib
        bad = cache.device(DEV)
        setattr(bad.struct, field, value)
        calls.append((status, lambda bad=bad: ctx._check(lib().sb_kv4_append(ctx._h, bad.struct, x.data_ptr(), 128, 64, x.data_ptr(), 128, 64, 2,
                                                                             starts.data_ptr(), lens.data_ptr(), 1))))
    for status, call in calls:
        with pytest.raises(SbError) as e:
            call()
        assert e.value.status == status
    ctx.sync()
