"""Requests' starts and lengths as the binding hands them to the library: one after the other in memory, or refused."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_17698_b200 import binding


def test_starts_and_lens_are_contiguous(monkeypatch):
    monkeypatch.setattr(binding, "_dev", lambda t: t.data_ptr())       # nothing is called: tensors on the CPU do
    cache = SimpleNamespace(struct=SimpleNamespace(requests=3))
    starts, lens = torch.arange(4, dtype=torch.int32), torch.full((3,), 20, dtype=torch.int32)
    assert binding.Context._kv8_rows(cache, starts, lens) == (starts.data_ptr(), lens.data_ptr())
    meta = torch.zeros(4, 2, dtype=torch.int32)
    both = torch.zeros(2, 7, dtype=torch.int32)
    assert binding.Context._kv8_rows(cache, both[1, :4], both[0, 4:]) == (both[1].data_ptr(), both[0, 4:].data_ptr())
    for s, n in [(starts, meta[:3, 1]), (meta[:, 0], lens), (starts, lens[:1].expand(3)), (torch.zeros(8, dtype=torch.int32)[::2], lens)]:
        with pytest.raises(ValueError):
            binding.Context._kv8_rows(cache, s, n)
