"""Ranks between the ones that the kernels are made for: what is padded takes no part in the result."""
import pytest
import torch

from test_gpu_lora import Case, _device, ctx  # noqa: F401  (ctx: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rank", [8, 16, 24, 40, 64, 72, 120, 128])
@pytest.mark.parametrize("new", [[2], [40], [200]])
def test_an_infinity_stays_one(ctx, new, rank, dtype):  # noqa: F811
    """With A and B positive an infinity of X is one of the whole row, at any rank."""
    case = Case(new, [0], 520, 72, rank, 1, dtype, scaled=False)
    case.adapters.a.abs_().clamp_min_(2.0 ** -10)
    case.adapters.b.abs_().clamp_min_(2.0 ** -10)
    x = _device(case.x)
    x[1, 5], x[0, 519] = float("inf"), float("-inf")
    out = ctx.lora_add(case.adapters, x, case.base, *case.args, out=torch.empty_like(case.base))
    ctx.sync()
    assert (out[1] == float("inf")).all() and (out[0] == float("-inf")).all() and torch.isfinite(out[2:].float()).all()


@pytest.mark.parametrize("rank", [8, 24, 72])
@pytest.mark.parametrize("new", [[2, 3], [40, 30]])
def test_infinities_stay_where_they_are(ctx, new, rank):  # noqa: F811
    """One infinity of X: every column is an infinity of the formula's sign, or NaN where its inner sums are of both signs."""
    case = Case(new, [0, 2], 128, 64, rank, 3)
    x = _device(case.x)
    case.adapters.a[1], case.adapters.b[1] = float("nan"), float("inf")
    x[0, 3], x[1] = float("inf"), float("nan")
    out = ctx.lora_add(case.adapters, x, case.base, *case.args, out=torch.empty_like(case.base))
    ctx.sync()
    signs = torch.from_numpy(case.a[0, :, 3]).sign() * torch.from_numpy(case.b[0]).sign() * float(case.scale[0])      # [out][rank]
    first = out[0].double().cpu()
    assert torch.equal(first == float("inf"), (signs > 0).all(1)) and torch.equal(first == float("-inf"), (signs < 0).all(1))
    assert not torch.isfinite(first).any() and torch.isnan(out[1].float()).all()
    case.x[:2] = 0
    case.check(out, slice(2, None))
