"""What the binding tells the library of a cache's page table."""
import pytest
import torch

from paper_2602_17698_b200 import binding


@pytest.fixture
def cache(monkeypatch):
    """A cache around a table, on the CPU (nothing is called)."""
    monkeypatch.setattr(binding, "_dev", lambda t: t.data_ptr())

    def make(table):
        kv = torch.zeros(8, 2, 16, 16, dtype=torch.int8)
        sc = torch.zeros(8, 2, 1, dtype=torch.bfloat16)
        return binding.Kv8Cache(kv, kv.clone(), sc, sc.clone(), table).struct
    return make


def test_rows_of_a_wider_table(cache):
    table = torch.zeros(3, 10, dtype=torch.int32)
    for view, stride, pages in [(table, 10, 10), (table[:, :4], 10, 4), (table[:, 2:3], 10, 1), (table[::2, :4], 20, 4),
                                (table[:1, :4].expand(5, 4), 0, 4), (table[0].expand(5, 10), 0, 10)]:
        s = cache(view)
        assert (s.table_stride, s.table_pages, s.requests, s.table) == (stride, pages, view.shape[0], view.data_ptr())
    for view in (table[:1, :4], table[2:, 5:9]):             # the stride of one row is never used
        assert cache(view).table_pages == 4


def test_refused_tables(cache):
    table = torch.zeros(3, 10, dtype=torch.int32)
    for bad in (table[:, ::2], table.t(), table[:, :0]):
        with pytest.raises(ValueError):
            cache(bad)
    with pytest.raises(TypeError):
        cache(table.long())
