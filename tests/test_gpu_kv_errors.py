"""What a cache's call reports says which cache it was."""
import re

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.fixture(scope="module")
def ctx():
    from paper_2602_17698_b200.binding import Context
    torch.cuda.set_device(0)
    c = Context()
    yield c
    c.close()


def _calls(ctx, bits):
    from paper_2602_17698_b200.binding import Kv4Cache, Kv8Cache
    cache = (Kv4Cache if bits == 4 else Kv8Cache).empty(4, 1, 16, 64, torch.zeros(1, 4, dtype=torch.int32, device=DEV))
    return cache, *(getattr(ctx, f"kv{bits}_{name}") for name in ("append", "read", "attention"))


@pytest.mark.parametrize("new", [1, 90])
def test_the_family_that_latched(ctx, new):
    """A request longer than its pages, by every call of both caches; NaN and a page that does not exist."""
    from paper_2602_17698_b200.binding import SbError
    found = {}
    for bits in (4, 8):
        cache, append, read, attention = _calls(ctx, bits)
        x, starts = torch.ones(new, 1, 64, dtype=torch.bfloat16, device=DEV), _ints(0, new)
        far = torch.full((1, 4), 9, dtype=torch.int32, device=DEV)
        gone = type(cache)(cache.k, cache.v, cache.k_scale, cache.v_scale, far, *([64] if bits == 4 else []))
        calls = [lambda: append(cache, x, x, starts, _ints(100), new), lambda: read(cache, starts, _ints(100), new, total=new),
                 lambda: attention(cache, x, starts, _ints(100), new, 64)]
        if new == 1:
            calls += [lambda: append(cache, x * float("nan"), x, starts, _ints(5), new), lambda: append(gone, x, x, starts, _ints(5), new),
                      lambda: attention(gone, x, starts, _ints(5), new, 64)]
        for call in calls:
            call()
            with pytest.raises(SbError) as e:
                ctx.sync()
            found.setdefault(bits, set()).add(re.search(r"family (\d+)", str(e.value)).group(1))
    assert len(found[4]) == 1 and len(found[8]) == 1 and found[4] != found[8]


@pytest.mark.parametrize("bits", [4, 8])
def test_a_prompt_that_is_refused(ctx, bits):
    """More tiles of query rows than 31 bits count."""
    from paper_2602_17698_b200.binding import SB_ERR_SHAPE, SbError, lib
    cache, *_ = _calls(ctx, bits)
    cache.struct.requests = 60000
    x, some = torch.ones(1, 1, 64, dtype=torch.bfloat16, device=DEV), _ints(*[0] * 8)
    with pytest.raises(SbError) as e:
        ctx._check(getattr(lib(), f"sb_kv{bits}_attention")(ctx._h, cache.struct, x.data_ptr(), 64, 64, 1, 1, some.data_ptr(), some.data_ptr(), 1 << 30, 64, 1.0, 0,
                                                            x.data_ptr(), 64, 64, None))
    assert e.value.status == SB_ERR_SHAPE and f"kv{bits} attention" in str(e.value)
