"""The quantised attention block as a long-running program uses it: calls of many sizes."""
import numpy as np
import pytest
import torch

import lowbit_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _block(ctx, fmt="nv", max_tokens=600):
    from paper_2602_17698_b200.binding import Kv8Cache
    from paper_2602_17698_b200.serving import QuantizedAttention, page_table
    rng = np.random.default_rng(2)
    hidden, heads, kv_heads, dim = 1000, 8, 2, 64
    w_qkv, w_o = (torch.from_numpy(ref.bf16(rng.standard_normal(s) * s[1] ** -0.5)).to(torch.bfloat16).to(DEV)
                  for s in (((heads + 2 * kv_heads) * dim, hidden), (hidden, heads * dim)))
    cache = Kv8Cache.empty(64, kv_heads, 16, dim, page_table([1000], 16, 64, DEV))
    torch.cuda.current_stream().synchronize()
    return QuantizedAttention(ctx, w_qkv, w_o, heads, kv_heads, dim, cache, max_tokens, fmt), torch.from_numpy(
        ref.bf16(rng.standard_normal((max_tokens, hidden)))).to(torch.bfloat16).to(DEV)


def _run(block, x, n):
    return block(x[:n], torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV), n, 1000)


@pytest.mark.parametrize("fmt", ["nv", "mx"])
def test_memory_does_not_grow_with_the_sizes_seen(fmt):
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    ctx = Context()
    block, x = _block(ctx, fmt)
    first = {n: _run(block, x, n).clone() for n in (1, 129, 600)}
    ctx.sync()
    held = torch.cuda.memory_allocated()
    for n in list(range(1, 600, 7)) + [600, 129, 1]:
        y = _run(block, x, n)
        if n in first:
            assert torch.equal(y, first[n])
        del y
    ctx.sync()
    # a call's own starts and lens are let go with it: at most a few of torch's 512-byte blocks may stay
    assert torch.cuda.memory_allocated() <= held + 4096
    with pytest.raises(ValueError):
        _run(block, torch.cat((x, x)), 601)
    ctx.close()
