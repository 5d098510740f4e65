"""Rotary positions by starts and lens without max_new: every request's rows are turned, as many as there are."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_17698_b200 import binding


def test_what_the_library_is_given(monkeypatch):
    """On the CPU, with the library's call replaced."""
    given = []
    monkeypatch.setattr(binding, "_dev", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(binding, "lib", lambda: SimpleNamespace(sb_rotary=lambda *a: given.append(a) or 0))
    ctx = object.__new__(binding.Context)
    ctx._h = None
    table, q = binding.RotaryTable(torch.ones(8)), torch.zeros(7, 2, 16)
    starts, lens = torch.tensor([0, 5, 7], dtype=torch.int32), torch.tensor([9, 2], dtype=torch.int32)
    ctx.rotary(table, q, starts=starts, lens=lens)
    ctx.rotary(table, q, None, starts, lens, 5)
    ctx.rotary(table, q, None, starts, lens, 0)
    ctx.rotary(table, q, positions=torch.arange(7, dtype=torch.int32))
    assert [a[-1] for a in given] == [7, 5, 0, 0]


@pytest.mark.gpu
def test_all_rows_are_turned():
    torch.cuda.set_device(0)
    ctx = binding.Context()
    table = binding.RotaryTable(binding.rotary_frequencies(64).cuda())
    q = torch.randn(41, 2, 64, device="cuda")
    starts, lens = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 40, 41], [100, 3]))
    got, _ = ctx.rotary(table, q, starts=starts, lens=lens, out=torch.zeros_like(q))
    want, _ = ctx.rotary(table, q, positions=torch.tensor([*range(60, 100), 2], dtype=torch.int32, device="cuda"), out=torch.zeros_like(q))
    ctx.sync()
    assert torch.equal(got, want) and not torch.equal(got, q)
    ctx.close()
