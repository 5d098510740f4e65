"""The 8-bit key/value cache: appending bit for bit, attention against 64 bits."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["int8", "e4m3"]


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


def _cache(kind, lens, heads, page, dim, rng, spare=3):
    per = max(1, max(-(-ln // page) for ln in lens))
    order = rng.permutation(per * len(lens) + spare)
    table = order[:per * len(lens)].reshape(len(lens), per).astype(np.int64)
    return ref.Cache(kind, per * len(lens) + spare, heads, page, dim, table, rng)


def _same(cache, dev):
    for side, (code, scale) in enumerate(((dev.k, dev.k_scale), (dev.v, dev.v_scale))):
        np.testing.assert_array_equal(scale.float().cpu().numpy(), cache.scale[side])
        np.testing.assert_array_equal(code.float().cpu().numpy(), cache.code[side])


def _tokens(T, heads, dim, rng, spread=1.0):
    return ref.bf16(rng.standard_normal((T, heads, dim)) * np.exp(spread * rng.standard_normal((T, 1, 1))))


def _device(x):
    return torch.from_numpy(x).to(torch.bfloat16).to(DEV)


# ---- appending --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past,new,heads,page,dim", [
    ([0], [1], 1, 16, 16), ([15], [1], 2, 16, 128), ([16], [1], 2, 16, 128), ([7, 0, 33], [1, 1, 1], 8, 64, 128),
    ([5, 40, 0, 100], [70, 0, 33, 1], 3, 48, 80), ([0, 3], [500, 16], 2, 32, 64), ([31, 1], [2, 40], 1, 128, 256), ([1], [300], 4, 16, 96)])
def test_append_is_exact(ctx, kind, past, new, heads, page, dim):
    rng = np.random.default_rng(sum(past) + 3 * sum(new) + dim)
    lens, starts = [p + n for p, n in zip(past, new)], _starts(new)
    cache = _cache(kind, lens, heads, page, dim, rng)
    dev = cache.device(DEV)
    k, v = _tokens(starts[-1], heads, dim, rng), _tokens(starts[-1], heads, dim, rng)
    for side, x in enumerate((k, v)):
        cache.append(side, x, starts, lens)
    for _ in range(2):                         # the second time changes nothing
        ctx.kv8_append(dev, _device(k), _device(v), _ints(starts), _ints(lens), max(new))
        ctx.sync()
        _same(cache, dev)


@pytest.mark.parametrize("kind", KINDS)
def test_a_block_that_fills_token_by_token(ctx, kind):
    """Scales that grow with larger tokens and stay with smaller ones; rows of K and V in one wider matrix."""
    rng = np.random.default_rng(9)
    cache = _cache(kind, [40, 40], 2, 32, 64, rng)
    dev = cache.device(DEV)
    size = np.exp(2 * rng.standard_normal(40))
    for step in range(33):
        lens, starts = [step + 1, step + 7], _starts([1, 1])
        qkv = ref.bf16(rng.standard_normal((2, 6 * 64)) * size[step])
        k, v = (qkv[:, i * 128:(i + 1) * 128].reshape(2, 2, 64) for i in (1, 2))
        d = _device(qkv)
        ctx.kv8_append(dev, d[:, 128:256].view(2, 2, 64), d[:, 256:].view(2, 2, 64), _ints(starts), _ints(lens), 1)
        for side, x in enumerate((k, v)):
            cache.append(side, x, starts, lens)
    ctx.sync()
    _same(cache, dev)


@pytest.mark.parametrize("kind", KINDS)
def test_zeros_and_extreme_sizes(ctx, kind):
    rng = np.random.default_rng(4)
    new, heads, dim = 80, 2, 128
    cache = _cache(kind, [new], heads, 16, dim, rng)
    dev = cache.device(DEV)
    x = ref.bf16(rng.standard_normal((new, heads, dim)))
    x[:16] = 0
    x[16:32] *= np.float32(2.0) ** -132                        # subnormal numbers
    x[32:48] = ref.bf16(x[32:48] * np.float32(2.0 ** 124))
    x[48:64, 0] = 0
    starts, lens = [0, new], [new]
    x = ref.bf16(x)
    for side in range(2):
        cache.append(side, x, starts, lens)
    ctx.kv8_append(dev, _device(x), _device(x), _ints(starts), _ints(lens), new)
    ctx.sync()
    _same(cache, dev)


@pytest.mark.parametrize("kind", KINDS)
def test_not_a_number_is_stored_as_zero_and_reported(ctx, kind):
    from paper_2602_17698_b200.binding import SB_ERR_NONFINITE, SbError
    rng = np.random.default_rng(4)
    cache = _cache(kind, [40], 1, 16, 64, rng)
    dev = cache.device(DEV)
    x = _tokens(40, 1, 64, rng, 0)
    x[3, 0, 5], x[20, 0, 6], x[20, 0, 7] = np.nan, np.inf, -np.inf
    ctx.kv8_append(dev, _device(x), _device(x), _ints([0, 40]), _ints([40]), 40)
    with pytest.raises(SbError) as e:
        ctx.sync()
    assert e.value.status == SB_ERR_NONFINITE
    for side in range(2):
        cache.append(side, x, [0, 40], [40])
    _same(cache, dev)
    assert cache.code[0][cache.table[0, 0], 0, 3, 5] == 0 and cache.code[0][cache.table[0, 1], 0, 4, 6] == cache.qmax
    ctx.sync()


@pytest.mark.parametrize("kind", KINDS)
def test_reading_back(ctx, kind):
    rng = np.random.default_rng(6)
    past, back, heads, dim = [0, 30, 7], [50, 0, 13], 2, 80
    lens, starts = [p + n for p, n in zip(past, back)], _starts(back)
    cache = _cache(kind, lens, heads, 32, dim, rng)
    k, v = ctx.kv8_read(cache.device(DEV), _ints(starts), _ints(lens), 50)
    ctx.sync()
    for side, x in enumerate((k, v)):
        for b in range(3):
            want = ref.bf16(cache.values(side, b, lens[b])[:, past[b]:].transpose(1, 0, 2))
            np.testing.assert_array_equal(x[starts[b]:starts[b + 1]].float().cpu().numpy(), want)


def test_requests_that_do_not_fit_are_skipped_and_reported(ctx):
    """Numbers on the device that do not fit: nothing is read or written outside, the others are served."""
    from paper_2602_17698_b200.binding import SB_ERR_INVALID, SbError
    rng = np.random.default_rng(8)
    heads, dim, page = 2, 64, 16
    good = [20, 40]
    cache = _cache("int8", good + [16], heads, page, dim, rng, spare=0)
    x, q = _tokens(20, heads, dim, rng), _tokens(20, 2 * heads, dim, rng)
    for case in range(6):
        dev = cache.device(DEV)
        lens, starts = [20, 40, 16], [0, 4, 8, 20]
        if case == 0: lens[2] = 1000                          # more tokens than pages
        if case == 1: lens[2] = 3                             # fewer tokens than new ones
        if case == 2: starts[3] = 21                          # past the dense rows
        if case == 3: starts[3] = 7                           # backwards
        if case == 4: dev.table[2, 0] = 10 ** 6               # no such page
        if case == 5: dev.table[2, 0] = -1
        before = [t.clone() for t in (dev.k, dev.v)]
        ctx.kv8_append(dev, _device(x), _device(x), _ints(starts), _ints(lens), 12)
        with pytest.raises(SbError) as e:
            ctx.sync()
        assert e.value.status == SB_ERR_INVALID
        for t, b, side in zip((dev.k, dev.v), before, range(2)):
            want = torch.from_numpy(cache.code[side]).to(torch.int8).to(DEV)
            assert torch.equal(t[cache.table[2]], want[cache.table[2]])
            assert not torch.equal(t, b)
        out = torch.full((20, 2 * heads, dim), 7.0, dtype=torch.bfloat16, device=DEV)
        ctx.kv8_attention(dev, _device(q), _ints(starts), _ints(lens), 12, 48, out=out)
        with pytest.raises(SbError) as e:
            ctx.sync()
        assert e.value.status == SB_ERR_INVALID
        assert (out[:8] != 7).any() and torch.isfinite(out.float()).all()


# ---- attention --------------------------------------------------------------------------------------------------

def _attend(ctx, kind, past, new, heads, group, page, dim, window=0, scale=None, qsize=1.0, max_len=None, seed=0, poison=True, wide=False,
            change=None):
    rng = np.random.default_rng(seed + sum(past) + 3 * sum(new) + dim + 11 * group)
    lens, starts = [p + n for p, n in zip(past, new)], _starts(new)
    cache = _cache(kind, lens, heads, page, dim, rng)
    if change:
        change(cache)
    dev = cache.device(DEV)
    if poison:
        # slots past a request's end hold anything: NaN codes, and NaN scales where no token shares them
        for b, ln in enumerate(lens):
            for p in range(ln, cache.table.shape[1] * page):
                pg, slot = int(cache.table[b, p // page]), p % page
                dev.k.view(torch.uint8)[pg, :, slot] = 0x7f
                dev.v.view(torch.uint8)[pg, :, slot] = 0xff
                if p % 16 == 0:
                    dev.k_scale[pg, :, slot // 16] = float("nan")
                    dev.v_scale[pg, :, slot // 16] = float("nan")
    T = starts[-1]
    q = ref.bf16(rng.standard_normal((T, heads * group, dim)) * qsize)
    qd, out = _device(q), None
    if wide:
        buf = torch.zeros(T, heads * group * dim + 64, dtype=torch.bfloat16, device=DEV)
        buf[:, :-64] = qd.view(T, -1)
        qd = buf[:, :-64].view(T, heads * group, dim)
        obuf = torch.full((T, heads * group + 2, dim + 8), 5.0, dtype=torch.bfloat16, device=DEV)
        out = obuf[:, :-2, :-8]
    sc = dim ** -0.5 if scale is None else scale
    out, lse = ctx.kv8_attention(dev, qd, _ints(starts), _ints(lens), max(new), max(lens) if max_len is None else max_len, scale=scale,
                                 window=window, out=out, want_lse=True)
    ctx.sync()
    want, wlse, mag, top, held = ref.attention(cache, q, starts, lens, sc, window)
    # the last rounding, 2^-8 of the result (bf16's unit roundoff); every weight rounded to fp16, 2^-11 of weight x |v| (and below
    # 2^-14 of the largest weight an absolute 2^-25 of it, under a scale of at most twice the largest
    # value scale); scores summed in fp32, 2^-20 of their terms'
    # magnitudes, which moves a weight by that much
    eps = 2.0 ** -20 * (top + 1)
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * eps[..., None]) * mag + 2.0 ** -24 * held + 1e-30
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
    lerr = np.abs(lse.double().cpu().numpy() - wlse)
    assert (lerr <= eps + 2.0 ** -21 * np.abs(wlse)).all(), float((lerr / eps).max())
    if wide:
        assert (obuf[:, -2:] == 5).all() and (obuf[:, :, -8:] == 5).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past,new,heads,group,page,dim", [
    ([0], [1], 1, 1, 16, 128), ([1], [1], 2, 4, 16, 64), ([15, 16, 17], [1, 1, 1], 2, 8, 16, 128), ([100, 0, 63], [1, 0, 1], 1, 5, 48, 80),
    ([500, 31, 32, 33], [1, 1, 1, 1], 4, 4, 64, 128), ([700], [1], 1, 12, 32, 256), ([90, 200], [1, 1], 2, 3, 128, 16)])
def test_one_token_per_request(ctx, kind, past, new, heads, group, page, dim):
    _attend(ctx, kind, past, new, heads, group, page, dim)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past,new,heads,group,page,dim", [
    ([40, 3], [5, 2], 2, 4, 16, 128), ([0], [33], 1, 2, 16, 64), ([17, 0, 64], [40, 70, 0], 2, 3, 32, 128), ([30], [20], 1, 7, 48, 256),
    ([0, 100], [130, 1], 1, 4, 64, 96), ([5], [150], 1, 8, 16, 128), ([0, 257], [300, 129], 2, 1, 64, 128)])
def test_drafts_and_prompts(ctx, kind, past, new, heads, group, page, dim):
    _attend(ctx, kind, past, new, heads, group, page, dim)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("window", [1, 2, 16, 50, 129])
@pytest.mark.parametrize("past,new", [([200, 10], [1, 1]), ([300, 0], [6, 9]), ([150, 0], [40, 140])])
def test_sliding_window(ctx, kind, window, past, new):
    _attend(ctx, kind, past, new, 2, 4, 32, 64, window=window)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_long_cache_in_many_chunks(ctx, kind, dim):
    _attend(ctx, kind, [9000, 1234], [1, 3], 1, 4, 64, dim, poison=False)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past,new,heads,group,dim,window", [
    ([3000], [70], 1, 4, 128, 0), ([2500, 10], [33, 65], 2, 3, 64, 0), ([1500], [257], 1, 1, 96, 0), ([4000, 0], [40, 64], 1, 4, 80, 700),
    ([0], [129], 1, 2, 128, 0), ([1111, 0, 127], [20, 0, 40], 2, 5, 128, 0)])
def test_chunks_of_prompts_behind_a_long_past(ctx, kind, past, new, heads, group, dim, window):
    _attend(ctx, kind, past, new, heads, group, 16, dim, window=window)


@pytest.mark.parametrize("max_len", [1, 1500, 10 ** 6])
def test_max_len_with_many_rows(ctx, max_len):
    _attend(ctx, "e4m3", [2900, 40], [30, 20], 1, 4, 32, 128, max_len=max_len)


@pytest.mark.parametrize("max_len", [1, 100, 2000, 3000])
def test_max_len_decides_nothing_but_the_chunks(ctx, max_len):
    _attend(ctx, "int8", [2900, 40], [2, 1], 1, 3, 100 // 16 * 16, 128, max_len=max_len, poison=False)


@pytest.mark.parametrize("kind", KINDS)
def test_strided_queries_and_outputs(ctx, kind):
    _attend(ctx, kind, [70, 20], [3, 40], 2, 2, 16, 128, wide=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("qsize", [1e-30, 1e-4, 30.0, 1e4])
def test_sizes_of_queries(ctx, kind, qsize):
    """From scores that are all equal to ones that pick a single key; fp16 alone would lose both ends."""
    _attend(ctx, kind, [300, 40], [1, 30], 1, 4, 16, 64, qsize=qsize, scale=0.125 if qsize < 1e3 else 1e-5)


@pytest.mark.parametrize("kind", KINDS)
def test_value_scales_of_very_different_sizes(ctx, kind):
    def change(cache):
        cache.scale[1] = ref.bf16(cache.scale[1] * np.exp(6 * np.random.default_rng(1).standard_normal(cache.scale[1].shape)))
        cache.scale[1][cache.table[0, 1]] = 0
        cache.scale[0][cache.table[0, 2]] = 0
    _attend(ctx, kind, [400, 60], [1, 20], 1, 4, 16, 128, change=change)


@pytest.mark.parametrize("kind", KINDS)
def test_a_cache_whose_values_are_zero(ctx, kind):
    def change(cache):
        cache.scale[1][:] = 0
    _attend(ctx, kind, [100], [2], 1, 2, 16, 128, change=change)


def test_offsets_beyond_32_bits(ctx):
    """Pages near the end of a cache of more than 2^32 bytes give what the same pages at its start give."""
    from paper_2602_17698_b200.binding import Kv8Cache
    rng = np.random.default_rng(2)
    cache = _cache("int8", [300, 70], 1, 64, 128, rng, spare=0)
    small = cache.device(DEV)
    n, pages = cache.code[0].shape[0], (1 << 32) // (64 * 128) + 5000
    big = [torch.empty(pages, 1, 64, 128, dtype=torch.int8, device=DEV) for _ in range(2)]
    scale = [torch.empty(pages, 1, 4, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for t, s, code, sc in zip(big, scale, (small.k, small.v), (small.k_scale, small.v_scale)):
        t[-n:], s[-n:] = code, sc
    far = Kv8Cache(big[0], big[1], scale[0], scale[1], small.table + (pages - n))
    for new in ([1, 1], [3, 40]):
        starts, lens = _starts(new), [300, 70]
        x, q = _device(_tokens(sum(new), 1, 128, rng)), _device(_tokens(sum(new), 4, 128, rng))
        outs = []
        for c in (small, far):
            ctx.kv8_append(c, x, x, _ints(starts), _ints(lens), max(new))
            outs.append((*ctx.kv8_attention(c, q, _ints(starts), _ints(lens), max(new), 300, want_lse=True),
                         *ctx.kv8_read(c, _ints(starts), _ints(lens), max(new))))
        ctx.sync()
        for a, b in zip(*outs):
            assert torch.equal(a, b)
    del far, big, t
    torch.cuda.empty_cache()


def test_same_sums_every_time_and_in_a_graph(ctx):
    """A captured step serves requests that grow: lengths and tables are read on the device."""
    from paper_2602_17698_b200.binding import Context
    rng = np.random.default_rng(3)
    heads, dim, page = 2, 128, 16
    cache = _cache("e4m3", [4000, 700], heads, page, dim, rng)
    x, q = _device(_tokens(2, heads, dim, rng)), _device(_tokens(2, 8, dim, rng))
    starts, lens = _ints([0, 1, 2]), _ints([3000, 600])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = Context(stream=side)
        dev, dev2 = cache.device(DEV), cache.device(DEV)
        out = torch.empty(2, 8, dim, dtype=torch.bfloat16, device=DEV)
        c.kv8_attention(dev, q, starts, lens, 1, 4000, out=out)           # the workspace grows outside the capture
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.kv8_append(dev, x, x, starts, lens, 1)
            c.kv8_attention(dev, q, starts, lens, 1, 4000, out=out)
        for _ in range(20):
            lens += 37
            graph.replay()
            c.kv8_append(dev2, x, x, starts, lens, 1)
            want, _ = c.kv8_attention(dev2, q, starts, lens, 1, 4000)
            c.sync()
            assert torch.equal(out, want)
        del graph
        c.close()


def test_nothing_new_is_nothing_done(ctx):
    rng = np.random.default_rng(3)
    cache = _cache("int8", [30], 1, 16, 64, rng)
    dev = cache.device(DEV)
    e = torch.empty(0, 1, 64, dtype=torch.bfloat16, device=DEV)
    launches = ctx.kernel_launches()
    ctx.kv8_append(dev, e, e, _ints([0, 0]), _ints([30]), 0)
    out, _ = ctx.kv8_attention(dev, e, _ints([0, 0]), _ints([30]), 0, 30)
    assert out.shape == (0, 1, 64) and ctx.kernel_launches() == launches
    ctx.sync()
    _same(cache, dev)


def test_refusals(ctx):
    from paper_2602_17698_b200.binding import Kv8Cache, SB_ERR_INVALID, SB_ERR_SHAPE, SbError
    rng = np.random.default_rng(3)
    dev = _cache("int8", [64], 2, 16, 64, rng).device(DEV)
    starts, lens = _ints([0, 2]), _ints([60])
    x, q = _device(_tokens(2, 2, 64, rng)), _device(_tokens(2, 6, 64, rng))
    launches = ctx.kernel_launches()

    def changed(**kw):
        c = Kv8Cache(dev.k, dev.v, dev.k_scale, dev.v_scale, dev.table)
        for k, v in kw.items():
            setattr(c.struct, k, v)
        return c
    odd = torch.zeros(2 * 130 + 1, dtype=torch.bfloat16, device=DEV)
    wide = torch.zeros(2, 2, 68, dtype=torch.bfloat16, device=DEV)[..., :64]
    for status, call in [
        (SB_ERR_INVALID, lambda: ctx.kv8_append(changed(type=2), x, x, starts, lens, 2)),
        (SB_ERR_INVALID, lambda: ctx.kv8_append(changed(k=None), x, x, starts, lens, 2)),
        (SB_ERR_INVALID, lambda: ctx.kv8_append(changed(pages=0), x, x, starts, lens, 2)),
        (SB_ERR_SHAPE, lambda: ctx.kv8_append(changed(page_tokens=24), x, x, starts, lens, 2)),
        (SB_ERR_SHAPE, lambda: ctx.kv8_append(changed(k=dev.k.data_ptr() + 8), x, x, starts, lens, 2)),
        (SB_ERR_SHAPE, lambda: ctx.kv8_append(dev, odd[1:257].view(2, 2, 64), x, starts, lens, 2)),
        (SB_ERR_SHAPE, lambda: ctx.kv8_append(dev, wide, x, starts, lens, 2)),
        (SB_ERR_INVALID, lambda: ctx.kv8_append(dev, x, x, starts, lens, -1)),
        (SB_ERR_SHAPE, lambda: ctx.kv8_attention(dev, _device(_tokens(2, 3, 64, rng)), starts, lens, 2, 64)),
        (SB_ERR_INVALID, lambda: ctx.kv8_attention(dev, q, starts, lens, 2, 0)),
        (SB_ERR_INVALID, lambda: ctx.kv8_attention(dev, q, starts, lens, 2, 64, window=-1)),
        (SB_ERR_INVALID, lambda: ctx.kv8_attention(dev, q, starts, lens, 2, 64, scale=float("nan"))),
        (SB_ERR_SHAPE, lambda: ctx.kv8_attention(dev, wide, starts, lens, 2, 64)),
        (SB_ERR_SHAPE, lambda: ctx.kv8_read(changed(dim=24), starts, lens, 2, out=(torch.zeros(2, 2, 24, dtype=torch.bfloat16, device=DEV),) * 2)),
    ]:
        with pytest.raises(SbError) as e:
            call()
        assert e.value.status == status, ctx
    for call in [lambda: Kv8Cache(dev.k.float(), dev.v, dev.k_scale, dev.v_scale, dev.table), lambda: Kv8Cache(dev.k, dev.v[:-1], dev.k_scale, dev.v_scale, dev.table),
                 lambda: Kv8Cache(dev.k, dev.v, dev.k_scale.float(), dev.v_scale, dev.table), lambda: Kv8Cache(dev.k, dev.v, dev.k_scale, dev.v_scale, dev.table.long()),
                 lambda: Kv8Cache(dev.k.transpose(1, 2), dev.v.transpose(1, 2), dev.k_scale, dev.v_scale, dev.table),
                 lambda: ctx.kv8_append(dev, x[:, :1], x[:, :1], starts, lens, 2), lambda: ctx.kv8_append(dev, x.float(), x.float(), starts, lens, 2),
                 lambda: ctx.kv8_append(dev, x, x, starts.long(), lens, 2), lambda: ctx.kv8_append(dev, x, x, starts[:1], lens, 2),
                 lambda: ctx.kv8_attention(dev, q[..., :32], starts, lens, 2, 64), lambda: ctx.kv8_attention(dev, q, starts, lens, 2, 64, out=q[:1])]:
        with pytest.raises((ValueError, TypeError)):
            call()
    assert ctx.kernel_launches() == launches
    ctx.sync()
