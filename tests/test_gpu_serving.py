"""The quantised attention block: the operators together, against the same block in plain form."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _plain(x, w, fmt, gx, gw):
    """bf16 product of two bf16 matrices (as fp32) that go through 4 bits."""
    vx = ref.fp4_values(*ref.fp4_quantize(x, fmt, gx)[::2], x.shape[1])
    vw = ref.fp4_values(*ref.fp4_quantize(w, fmt, gw)[::2], w.shape[1])
    return ref.bf16(vx @ vw.T)


@pytest.mark.parametrize("fmt,kind", [("nv", "int8"), ("mx", "e4m3")])
def test_prompts_and_decode_steps(fmt, kind):
    from paper_2602_17698_b200.binding import Context, Kv8Cache
    from paper_2602_17698_b200.serving import QuantizedAttention, page_table, tensor_scale
    torch.cuda.set_device(0)
    ctx = Context()
    rng = np.random.default_rng(7)
    hidden, heads, kv_heads, dim, page = 256, 8, 2, 64, 16
    w_qkv = ref.bf16(rng.standard_normal(((heads + 2 * kv_heads) * dim, hidden)) * hidden ** -0.5)
    w_o = ref.bf16(rng.standard_normal((hidden, heads * dim)) * (heads * dim) ** -0.5)
    prompts, pages = [40, 3, 17], 16
    table = page_table([p + 4 for p in prompts], page, pages, DEV)
    cache = Kv8Cache.empty(pages, kv_heads, page, dim, table, torch.int8 if kind == "int8" else torch.float8_e4m3fn)
    host = ref.Cache(kind, pages, kv_heads, page, dim, table.cpu().numpy().astype(np.int64), rng)
    dq, do = (torch.from_numpy(w).to(torch.bfloat16).to(DEV) for w in (w_qkv, w_o))
    gx, go = (0.5, 0.0625) if fmt == "nv" else (None, None)
    scale = [None if g is None else torch.tensor([g], device=DEV) for g in (gx, go)]
    block = QuantizedAttention(ctx, dq, do, heads, kv_heads, dim, cache, sum(prompts), fmt, *scale)
    gq, gw = (float(tensor_scale(w)) if fmt == "nv" else None for w in (dq, do))
    done = [0, 0, 0]
    for new in (prompts, [1, 1, 1], [2, 0, 1]):
        starts = [0] + list(np.cumsum(new))
        done = [a + b for a, b in zip(done, new)]
        x = ref.bf16(rng.standard_normal((starts[-1], hidden)))
        y = block(torch.from_numpy(x).to(torch.bfloat16).to(DEV), torch.tensor(starts, dtype=torch.int32, device=DEV),
                  torch.tensor(done, dtype=torch.int32, device=DEV), max(new), 64)
        qkv = block.qkv[:starts[-1]].float().cpu().numpy()
        att = block.att[:starts[-1]].float().cpu().numpy()
        ctx.sync()
        # step by step on what the step before left, so that a rounding on the brink of the next step's
        # grid stays in its own step: products to one bf16 rounding and fp32 sums, the cache exactly
        want = _plain(x, w_qkv, fmt, gx, gq)
        np.testing.assert_allclose(qkv, want, rtol=2.0 ** -7, atol=1e-5)
        nq, nk = heads * dim, kv_heads * dim
        q, k, v = (t.reshape(len(x), -1, dim) for t in (qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]))
        host.append(0, k, starts, done)
        host.append(1, v, starts, done)
        for b, n in enumerate(done):
            for side, code, sc in ((0, cache.k, cache.k_scale), (1, cache.v, cache.v_scale)):
                p = np.arange(n)
                pg, slot = host.table[b, p // page], p % page
                np.testing.assert_array_equal(code.float().cpu().numpy()[pg, :, slot], host.code[side][pg, :, slot])
                np.testing.assert_array_equal(sc.float().cpu().numpy()[pg, :, slot // 16], host.scale[side][pg, :, slot // 16])
        out, _, mag, top, held = ref.attention(host, q, starts, done, dim ** -0.5, 0)
        tol = 2.0 ** -8 * np.abs(out) + (2.0 ** -11 + 2.0 ** -19 * (top + 1)[..., None]) * mag + 2.0 ** -24 * held + 1e-30
        assert (np.abs(att - out) <= tol).all()
        want = _plain(att.reshape(len(x), -1), w_o, fmt, go, gw)
        np.testing.assert_allclose(y.float().cpu().numpy(), want, rtol=2.0 ** -7, atol=1e-5)
    ctx.close()


def test_the_example_runs(capsys):
    from paper_2602_17698_b200 import serving
    torch.cuda.set_device(0)
    serving.main()
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 4
    for line in lines:
        # 4-bit inputs and weights: each about 0.1 off (uniform inside a binade of three steps), twice
        # per product, two products in a row
        assert 0.01 < float(line.split("block ")[1].split()[0]) < 0.4, line


def test_page_table_refuses_what_does_not_fit():
    from paper_2602_17698_b200.serving import page_table
    assert page_table([1, 33], 16, 4, "cpu").tolist() == [[0, 0, 0], [1, 2, 3]]
    with pytest.raises(ValueError):
        page_table([1, 33], 16, 3, "cpu")
