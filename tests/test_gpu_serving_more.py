"""The quantised attention block with rotary positions, adapters and a 4-bit cache: the operators together, step by step against plain forms."""
import numpy as np
import pytest
import torch

import lowbit_reference as low
import more_reference as ref
from test_gpu_serving import _plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _cuda(x, dtype=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(dtype).to(DEV)


@pytest.mark.parametrize("busy", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_prompts_and_decode_steps(busy, interleaved):
    """busy: the block has a stream of its own, which is behind."""
    from paper_2602_17698_b200.binding import Context, Kv4Cache, LoraAdapters, RotaryTable, rotary_frequencies
    from paper_2602_17698_b200.serving import QuantizedAttention, page_table, tensor_scale
    torch.cuda.set_device(0)
    stream = torch.cuda.Stream() if busy else None
    ctx = Context(stream=stream)
    rng = np.random.default_rng(7)
    hidden, heads, kv_heads, dim, page, rank = 256, 8, 2, 64, 16, 8
    nq, nk = heads * dim, kv_heads * dim
    w_qkv = low.bf16(rng.standard_normal((nq + 2 * nk, hidden)) * hidden ** -0.5)
    w_o = low.bf16(rng.standard_normal((hidden, nq)) * nq ** -0.5)
    lo = {n: (low.bf16(rng.standard_normal((3, rank, w.shape[1])) * w.shape[1] ** -0.5), low.bf16(rng.standard_normal((3, w.shape[0], rank)) * 0.2),
              rng.uniform(0.5, 1, 3).astype(np.float32)) for n, w in (("qkv", w_qkv), ("o", w_o))}
    prompts, pages = [40, 3, 17], 16
    table = page_table([p + 4 for p in prompts], page, pages, DEV)
    k_head, v_head = torch.tensor([0.5, 2.0], device=DEV), torch.tensor([1.0, 0.25], device=DEV)
    cache = Kv4Cache.empty(pages, kv_heads, page, dim, table, k_head, v_head)
    host = ref.Cache4(pages, kv_heads, page, dim, table.cpu().numpy().astype(np.int64), rng)
    host.head = [k_head.cpu().numpy(), v_head.cpu().numpy()]
    freq = rotary_frequencies(48, 5000.0, "parts", 4.0, trained=64)
    dq, do = _cuda(w_qkv), _cuda(w_o)
    gx, go = 0.5, 0.0625
    block = QuantizedAttention(ctx, dq, do, heads, kv_heads, dim, cache, sum(prompts), "nv", *(torch.tensor([g], device=DEV) for g in (gx, go)),
                               rotary=RotaryTable(freq.to(DEV), interleaved, 1.125),
                               **{n + "_adapters": LoraAdapters(_cuda(a), _cuda(b), _cuda(s, torch.float32)) for n, (a, b, s) in lo.items()})
    gq, gw = float(tensor_scale(dq)), float(tensor_scale(do))
    done, ids = [0, 0, 0], [2, -1, 0]
    for new in (prompts, [1, 1, 1], [2, 0, 1]):
        starts = [0] + list(np.cumsum(new))
        done = [a + b for a, b in zip(done, new)]
        x = low.bf16(rng.standard_normal((starts[-1], hidden)))
        if busy:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(5_000_000)
        y = block(_cuda(x), torch.tensor(starts, dtype=torch.int32, device=DEV), torch.tensor(done, dtype=torch.int32, device=DEV), max(new), 64,
                  ids=torch.tensor(ids, dtype=torch.int32, device=DEV)).clone()
        torch.cuda.synchronize()
        qkv, att = (t[:starts[-1]].float().cpu().numpy() for t in (block.qkv, block.att))
        ctx.sync()
        # on what the step before left: products to one bf16 rounding and fp32 sums, then the adapters' sum to another, positions to a third
        pos = np.concatenate([np.arange(n - m, n) for n, m in zip(done, new)])

        def projected(x, w, gx, gw, name):
            plain = _plain(x, w, "nv", gx, gw)
            want, second, first = ref.lora(x, plain, *lo[name], ids, starts)
            return want, 2.0 ** -7 * np.abs(plain) + 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * second + 2.0 ** -18 * first + 1e-5

        want, tol = projected(x, w_qkv, gx, gq, "qkv")
        for part, n in ((slice(0, nq), heads), (slice(nq, nq + nk), kv_heads)):
            w, t = (v[:, part].reshape(len(x), n, dim) for v in (want, tol))
            turned, _ = ref.rotary(w, pos, freq.numpy(), interleaved, 1.125)
            spread, size = np.abs(ref.rotary(t, pos, freq.numpy(), interleaved, 1.125)[0]), ref.rotary(t, pos, freq.numpy(), interleaved, 1.125)[1]
            t = np.where(size > 0, size, spread) + 2.0 ** -8 * np.abs(turned) + 1e-5
            assert (np.abs(qkv[:, part].reshape(w.shape) - turned) <= t).all()
        assert (np.abs(qkv - want)[:, nq + nk:] <= tol[:, nq + nk:]).all()
        q, k, v = (t.reshape(len(x), -1, dim) for t in (qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]))
        host.append(0, k, starts, done)
        host.append(1, v, starts, done)
        for b, n in enumerate(done):
            p = np.arange(n)
            pg, slot = host.table[b, p // page], p % page
            for side, code, sc in ((0, cache.k, cache.k_scale), (1, cache.v, cache.v_scale)):
                hq, hs = host.bytes(side)
                np.testing.assert_array_equal(code.cpu().numpy()[pg, :, slot], hq[pg, :, slot])
                np.testing.assert_array_equal(sc.cpu().numpy()[pg, :, slot], hs[pg, :, slot])
        out, _, mag, top, held = ref.attention(host, q, starts, done, dim ** -0.5, 0)
        tol = 2.0 ** -8 * np.abs(out) + (2.0 ** -11 + 2.0 ** -19 * (top + 1)[..., None]) * mag + 2.0 ** -31 * held + 1e-30
        assert (np.abs(att - out) <= tol).all()
        want, tol = projected(att.reshape(len(x), -1), w_o, go, gw, "o")
        assert (np.abs(y.float().cpu().numpy() - want) <= tol).all()
    ctx.close()


def test_an_8_bit_cache_and_no_adapters_called():
    """Options that are off change nothing: the block of before, with its hook."""
    from paper_2602_17698_b200.binding import Context, Kv8Cache, LoraAdapters
    from paper_2602_17698_b200.serving import QuantizedAttention, page_table
    torch.cuda.set_device(0)
    ctx = Context()
    g = torch.Generator(DEV).manual_seed(1)
    w_qkv, w_o = torch.randn(6 * 64, 128, device=DEV, generator=g).bfloat16() * 0.1, torch.randn(128, 256, device=DEV, generator=g).bfloat16() * 0.1
    x = torch.randn(30, 128, device=DEV, generator=g).bfloat16()
    starts, lens = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, 30], [30]))
    adapters = LoraAdapters(torch.ones(1, 8, 128, device=DEV).bfloat16(), torch.ones(1, 384, 8, device=DEV).bfloat16())
    ys = []
    for more in ({}, {"qkv_adapters": adapters}):
        cache = Kv8Cache.empty(4, 1, 16, 64, page_table([30], 16, 4, DEV))
        block = QuantizedAttention(ctx, w_qkv, w_o, 4, 1, 64, cache, 30, **more)
        ys.append(block(x, starts, lens, 30, 30, rotate=lambda q, k: q.mul_(0.5)).clone())
    ids = torch.tensor([0], dtype=torch.int32, device=DEV)
    other = block(x, starts, lens, 30, 30, rotate=lambda q, k: q.mul_(0.5), ids=ids)
    ctx.sync()
    assert torch.equal(*ys) and not torch.equal(ys[0], other)
    with pytest.raises(ValueError):
        QuantizedAttention(ctx, w_qkv, w_o, 4, 1, 64, cache, 30, o_adapters=adapters)
    ctx.close()


@pytest.mark.parametrize("argv", [["--cache", "4"], ["--rotary"], ["--adapters", "2"], ["--cache", "4", "--rotary", "--adapters", "3"]])
def test_the_example_runs(argv, capsys):
    from paper_2602_17698_b200 import serving
    torch.cuda.set_device(0)
    serving.main(argv)
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 4
    for line in lines:
        assert 0.01 < float(line.split("block ")[1].split()[0]) < 0.6, line
