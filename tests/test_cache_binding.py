"""The key-value cache's binding: what it tells the library of its arguments, and what it refuses before the library is called.
Nothing is launched; tensors are stand-ins that say they lie on the GPU."""
from types import SimpleNamespace

import pytest
import torch

from paper_2302_12510_b200 import binding

CACHE = SimpleNamespace(heads=2)


class Table:
    """A host tensor that passes for one of the device."""

    def __init__(self, t):
        self.t, self.dtype, self.is_cuda, self.shape = t, t.dtype, True, t.shape

    def __getattr__(self, name):
        return getattr(self.t, name)


def batch(table, **more):
    return binding._cache_batch(CACHE, Table(table), 8, 4, None, **more)


INTS = torch.arange(40, dtype=torch.int32)


@pytest.mark.parametrize("table", [INTS[:10].view(1, 10).expand(4, 10), INTS[:1].view(1, 1).expand(4, 1), INTS.unfold(0, 10, 3),
                                   INTS.unfold(0, 10, 9)], ids=["expanded", "expanded column", "sliding", "one shared entry"])
def test_tables_whose_rows_overlap_are_refused(table):
    with pytest.raises(ValueError):
        batch(table)


@pytest.mark.parametrize("table,stride", [(INTS.view(4, 10), 10), (INTS.view(4, 10)[:, 3:8], 10), (INTS.view(4, 10)[::2], 20), (INTS[:10].view(1, 10), 10),
                                          (INTS[:10].expand(1, 10), 10), (INTS.view(4, 10)[:1, 2:5], 3), (INTS.view(4, 10)[:, 3:4], 10),
                                          (INTS[:0].view(0, 10), 10), (INTS.view(4, 10)[:, :0], 10)])
def test_every_row_of_a_table_lies_in_it(table, stride):
    b = batch(table)
    assert (b.sequences, b.max_pages) == tuple(table.shape) and b.table_stride == stride and (b.table or 0) == table.data_ptr()
    if table.numel() > 0:
        last = (b.sequences - 1) * b.table_stride + b.max_pages - 1 + table.storage_offset()
        assert last < table.untyped_storage().nbytes() // 4
