"""What a kernel writes is what the next one, resident before it has ended, reads: the same buffers again and again with new contents, so that
anything an earlier launch left in a cache would show."""
import pytest
import torch

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
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _turn(dim):
    from paper_2602_17698_b200.binding import RotaryTable, rotary_frequencies
    return RotaryTable(rotary_frequencies(dim).to(DEV))


@pytest.mark.parametrize("new", [[1] * 200, [700, 1, 900, 33]])
def test_append_behind_rotary_in_place(ctx, new):
    """The cache's bytes and what is read back, against the same calls with a wait between them."""
    from paper_2602_17698_b200.binding import Kv4Cache
    from paper_2602_17698_b200.serving import page_table
    T, heads, dim, lens = sum(new), 8, 128, [n + 70 for n in new]
    table = page_table(lens, 16, sum(-(-n // 16) for n in lens), DEV)
    caches = [Kv4Cache.empty(int(table.max()) + 1, heads, 16, dim, table) for _ in range(2)]
    starts, ln, turn = _ints([0] + torch.tensor(new).cumsum(0).tolist()), _ints(lens), _turn(dim)
    qkv = torch.empty(T, 6 * heads * dim, dtype=torch.bfloat16, device=DEV)
    fresh = [torch.randn(qkv.shape, device=DEV).bfloat16() for _ in range(3)]
    q, k, v = (qkv[:, i * heads * dim:j * heads * dim].unflatten(1, (-1, dim)) for i, j in ((0, 4), (4, 5), (5, 6)))
    read = [torch.empty(T, heads, dim, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    for i in range(30):
        for wait, cache in enumerate(caches):
            qkv.copy_(fresh[i % 3]).mul_(1 + i)
            ctx.rotary(turn, q, k, starts, ln, max(new))
            if wait:
                ctx.sync()
            ctx.kv4_append(cache, k, v, starts, ln, max(new))
            if wait:
                ctx.sync()
            ctx.kv4_read(cache, starts, ln, max(new), out=read[2 * wait:2 * wait + 2])
        ctx.sync()
        for name in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(getattr(caches[0], name), getattr(caches[1], name))
        assert torch.equal(read[0], read[2]) and torch.equal(read[1], read[3])


@pytest.mark.parametrize("new,columns", [([1] * 64, 512), ([3, 16, 1, 0, 9] * 12, 512), ([700, 90, 1, 300], 512), ([700, 90, 1, 300], 500), ([700, 90, 1, 300], 502)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_adapters_behind_rotary_in_place(ctx, new, columns, dtype):
    """Both of X and base are written by the kernel ahead; `columns` of `out`: rows of base aligned to 16, 8 and 4 bytes (bf16)."""
    from paper_2602_17698_b200.binding import LoraAdapters
    T, inner, n = sum(new), 1024, 5
    starts, ids = _ints([0] + torch.tensor(new).cumsum(0).tolist()), _ints([i % (n + 1) - 1 for i in range(len(new))])
    adapters = LoraAdapters(torch.randn(n, 16, inner, device=DEV).bfloat16(), torch.randn(n, columns, 16, device=DEV).bfloat16())
    turn, at = _turn(64), _ints(list(range(T)))
    small = _turn(2)
    x, base = torch.empty(T, inner, dtype=torch.bfloat16, device=DEV), torch.empty(T, columns, dtype=dtype, device=DEV)
    fresh = [(torch.randn(x.shape, device=DEV).bfloat16(), torch.randn(base.shape, device=DEV).to(dtype)) for _ in range(3)]
    got = []
    for i in range(30):
        for wait in range(2):
            x.copy_(fresh[i % 3][0]).mul_(1 + i)
            base.copy_(fresh[i % 3][1]).mul_(1 + i)
            for order in ((x, 64, turn), (base, 2, small))[::1 if i & 1 else -1]:
                ctx.rotary(order[2], order[0].unflatten(1, (-1, order[1])), positions=at)
            if wait:
                ctx.sync()
            got.append(ctx.lora_add(adapters, x, base, ids, starts, max(new)).clone())
        ctx.sync()
        assert torch.equal(*got)
        got.clear()


@pytest.mark.parametrize("ahead", ["kernel", "copy", "fill", "two streams"])
def test_captured_behind_other_streams(ahead):
    """A graph in which the context's stream follows others' kernels, copies and fills, and others follow it, against the same calls one by one."""
    from paper_2602_17698_b200.binding import Context, Kv4Cache, LoraAdapters
    torch.cuda.set_device(0)
    main, other, side = (torch.cuda.Stream() for _ in range(3))
    T, heads, dim, R = 300, 2, 64, 3
    starts, lens, ids = _ints([0, 130, 131, T]), _ints([200, 31, 169]), _ints([1, -1, 0])
    table = torch.arange(3 * 13, dtype=torch.int32, device=DEV).view(3, 13)
    turn = _turn(dim)
    adapters = LoraAdapters(torch.randn(2, 24, heads * dim, device=DEV).bfloat16(), torch.randn(2, 70, 24, device=DEV).bfloat16())
    source, plus = torch.empty(T, heads, dim, dtype=torch.bfloat16, device=DEV), torch.empty(T, heads, dim, dtype=torch.bfloat16, device=DEV)

    class Run:
        def __init__(self):
            self.ctx = Context(stream=side)
            self.x = torch.empty_like(source)
            self.base = torch.zeros(T, 70, dtype=torch.bfloat16, device=DEV)
            self.cache = Kv4Cache.empty(39, heads, 16, dim, table)
            self.out, self.sum = torch.empty_like(source), torch.empty_like(source)

        def step(self):
            main.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(main):
                if ahead == "fill":
                    self.x.zero_()
                else:
                    self.x.copy_(source)
                if ahead == "kernel":
                    self.x.mul_(2)
            if ahead == "two streams":
                other.wait_stream(main)
                with torch.cuda.stream(other):
                    self.x[100:].add_(plus[100:])
                with torch.cuda.stream(main):
                    self.x[:100].mul_(3)
                side.wait_stream(other)
            side.wait_stream(main)
            with torch.cuda.stream(side):
                c = self.ctx
                c.rotary(turn, self.x, None, starts, lens, 200)
                c.kv4_append(self.cache, self.x, self.x, starts, lens, 200)
                c.kv4_attention(self.cache, self.x, starts, lens, 200, 200, out=self.out)
                c.lora_add(adapters, self.x.flatten(1), self.base, ids, starts, 200)
            main.wait_stream(side)
            with torch.cuda.stream(main):
                torch.add(self.out, self.x, out=self.sum)
            torch.cuda.current_stream().wait_stream(main)

    def new():
        source.copy_(torch.randn(source.shape, device=DEV))
        plus.copy_(torch.randn(source.shape, device=DEV))

    plain, captured = Run(), Run()
    new()
    torch.cuda.synchronize()
    captured.step()
    torch.cuda.synchronize()
    captured.base.zero_()
    graph, at = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=at):
        captured.step()
    for _ in range(8):
        new()
        torch.cuda.synchronize()
        plain.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("x", "base", "out", "sum"):
            assert torch.equal(getattr(plain, name), getattr(captured, name)), name
        assert torch.equal(plain.cache.k, captured.cache.k) and torch.equal(plain.cache.v_scale, captured.cache.v_scale)
    del graph
    for r in (plain, captured):
        r.ctx.sync()
        r.ctx.close()
