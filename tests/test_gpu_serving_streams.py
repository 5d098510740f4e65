"""The quantised attention block on a stream of its own, made and called while torch's current stream is another."""
import numpy as np
import pytest
import torch

from test_gpu_serving_workspaces import DEV, _block, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("busy", ["the current stream", "the block's stream", "both"])
def test_a_stream_of_its_own(busy):
    """Whichever stream is behind: the block's own work (the weights' tensor scales, what `rotate` does) is in order, and so are its
    inputs and its result with what the current stream does before and after."""
    from paper_2602_17698_b200.binding import Context
    from paper_2602_17698_b200.serving import QuantizedAttention
    torch.cuda.set_device(0)
    plain = Context()
    block, x = _block(plain)
    rng = np.random.default_rng(2)
    hidden, heads, kv_heads, dim = 1000, 8, 2, 64
    w_qkv, w_o = (torch.randn(s, device=DEV, generator=torch.Generator(DEV).manual_seed(i)).mul_(s[1] ** -0.5).bfloat16()
                  for i, s in enumerate((((heads + 2 * kv_heads) * dim, hidden), (hidden, heads * dim))))
    starts, lens = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, 300], [300]))

    def rotate(q, k):
        q.mul_(0.5)
        k.mul_(-1.0)

    def make(ctx):
        return QuantizedAttention(ctx, w_qkv, w_o, heads, kv_heads, dim, block.cache, 600)
    want = make(plain)(x[:300], starts, lens, 300, 1000, rotate=rotate).clone()
    plain.sync()
    stream = torch.cuda.Stream()
    ctx = Context(stream=stream)
    torch.cuda.synchronize()

    def wait():
        if busy != "the block's stream":
            torch.cuda._sleep(20_000_000)
        if busy != "the current stream":
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)
    wait()
    own = make(ctx)
    torch.cuda.synchronize()
    wait()
    late = x[:300] * 1                                       # an input that the current stream has yet to make
    got = own(late, starts, lens, 300, 1000, rotate=rotate).clone()
    del late
    torch.full((300, hidden), 7.0, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    plain.close()
    ctx.close()
