"""Many rows of few requests among slots without rows or with one: the work is that of the rows."""
import pytest
import torch

from test_gpu_lora import Case, _device, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [[0] * 300 + [17], [40] + [0] * 2000 + [65, 1], [1] * 127 + [17], [1] * 100 + [200] + [0, 1] * 40, [64] * 5 + [0] * 9])
def test_sizes(ctx, new, dtype):  # noqa: F811
    case = Case(new, [i % 4 - 1 for i in range(len(new) - 1)] + [2], 600, 200, 24, 3, dtype)
    out = torch.full_like(case.base, 9.0)
    ctx.lora_add(case.adapters, _device(case.x), case.base, *case.args, out=out)
    ctx.sync()
    case.check(out)


def test_the_time_is_the_rows(ctx):  # noqa: F811
    """64 rows beside 20000 empty slots: a quarter of a millisecond, where a block for each slot and part would take a third of a second."""
    case = Case([0] * 20000 + [64], [0] * 20001, 2048, 4096, 16, 1)
    x, out = _device(case.x), torch.empty_like(case.base)
    ctx.lora_add(case.adapters, x, case.base, *case.args, out=out)
    ctx.sync()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record(ctx.stream)
    ctx.lora_add(case.adapters, x, case.base, *case.args, out=out)
    end.record(ctx.stream)
    ctx.sync()
    case.check(out)
    assert begin.elapsed_time(end) < 20
