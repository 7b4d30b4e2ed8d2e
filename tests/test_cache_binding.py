"""The key-value cache's binding: what it tells the library of its arguments, and what it refuses before the library is called.
Nothing is launched; tensors are stand-ins that say they lie on the GPU."""
import weakref
from types import SimpleNamespace

import pytest
import torch

from paper_2302_12510_b200 import binding

CACHE = SimpleNamespace(heads=2)


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    """The stand-ins' device is the current one."""
    now = [0]
    monkeypatch.setattr(binding, "_raw_device", lambda: now[0])
    return now


class Table:
    """A host tensor that passes for one of a device."""

    def __init__(self, t, device="cuda:0"):
        self.t, self.dtype, self.is_cuda, self.shape, self.device = t, t.dtype, True, t.shape, torch.device(device)

    def get_device(self):
        return self.device.index

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


# ---------------------------------------------------------------- whole numbers that the library takes in 32 bits

@pytest.mark.parametrize("window,want", [(0, 0), (16, 16), (2**31 - 1, 2**31 - 1), (2**31, 2**31 - 1), (2**32 + 16, 2**31 - 1), (2**40, 2**31 - 1), (-1, -1)])
def test_a_window_is_not_cut(window, want):
    assert batch(INTS.view(4, 10), window=window).window == want
    assert Calls().attention(window=window)[-4] == want


@pytest.mark.parametrize("bad", [2**31, 2**32 + 4, -2**31 - 1, -2**32 + 4])
def test_other_numbers_beyond_32_bits_are_refused(bad):
    table, calls = Table(INTS.view(4, 10)), Calls()
    makes = [lambda: binding._cache_batch(CACHE, table, 8, bad, None), lambda: binding.KVCache(0, bad, 1, 64), lambda: binding.KVCache(0, 16, bad, 64),
             lambda: binding.KVCache(0, 16, 1, bad), lambda: calls.write(top=bad), lambda: binding._cache_batch(CACHE, table, bad, 4, None)]
    if bad < 0:
        makes += [lambda: batch(INTS.view(4, 10), window=bad), lambda: calls.attention(window=bad), lambda: binding._cache_batch(CACHE, table, 8, 4, bad)]
    for make in makes:
        with pytest.raises(ValueError):
            make()
    # (max_new bounds what there is: any number at or above it)
    assert binding._cache_batch(CACHE, table, 8, 4, 2**40).max_new == 8


class Calls:
    """The calls with a library that only notes its arguments."""

    def __init__(self):
        self.cache = SimpleNamespace(heads=2, dim=64, page=16, ref=None, device=0)
        self.plan = binding.CachePlan.__new__(binding.CachePlan)
        self.plan.__dict__.update(T=3, q_heads=4, ref=None, address=0, page=16, heads=2, device=0, _ws_bytes={64: 64})
        self.tensor = lambda *shape, device="cuda:0": Table(torch.zeros(shape, dtype=torch.bfloat16), device)

    def noted(self, name, call):
        seen, lib = [], binding.lib
        binding.lib = SimpleNamespace(**{name: lambda *args: seen.append(args) or 0})
        try:
            call()
        finally:
            binding.lib = lib
        return seen[0]

    def attention(self, q=None, out=None, **more):
        q, out = q or self.tensor(3, 4, 64), out or self.tensor(3, 4, 64)
        return self.noted("dybit_cache_attention", lambda: binding.dybit_cache_attention(q, self.cache, self.plan, out=out, stream=0,
                                                                                         ws=Table(torch.zeros(4096, dtype=torch.uint8)), **more))

    def write(self, **more):
        k = self.tensor(3, 2, 64)
        return self.noted("dybit_cache_write", lambda: binding.dybit_cache_write(self.cache, k, k, self.plan, stream=0, **more))


# ---------------------------------------------------------------- what a plan keeps

def test_a_plan_keeps_what_its_launch_reads():
    # tensors made for the call alone: on another stream than their own their memory could be another's before the launch has read them
    made = [Table(INTS.view(4, 10)), Table(torch.arange(5, dtype=torch.int32)), Table(torch.full((4,), 9, dtype=torch.int32))]
    alive, lib = [weakref.ref(t) for t in made], binding.lib
    binding.lib = SimpleNamespace(dybit_cache_plan_bytes=lambda *args: 64, dybit_cache_plan=lambda *args: 0)
    try:
        plan = binding.CachePlan(SimpleNamespace(heads=2, page=16, ref=None), *made, 4, buffer=Table(torch.zeros(64, dtype=torch.uint8)), stream=0)
    finally:
        binding.lib = lib
    del made
    assert all(ref() is not None for ref in alive)
    del plan
    assert all(ref() is None for ref in alive)


# ---------------------------------------------------------------- devices

def test_tensors_of_other_devices_are_refused(current_device):
    calls, far = Calls(), lambda *shape, dtype=torch.bfloat16: Table(torch.zeros(shape, dtype=dtype), "cuda:1")
    calls.attention(), calls.write()
    ints = [Table(INTS.view(4, 10)), Table(INTS[:5]), Table(INTS[:4])]
    plan = lambda *t, **more: binding.dybit_cache_plan(calls.cache, *t, 8, 4, stream=0, **more)
    refused = [lambda: calls.attention(q=far(3, 4, 64)), lambda: calls.attention(out=far(3, 4, 64)),
               lambda: calls.attention(lse=far(3, 4, dtype=torch.float32)), lambda: plan(ints[0], Table(INTS[:5], "cuda:1"), ints[2]),
               lambda: plan(*ints[:2], Table(INTS[:4], "cuda:1")), lambda: plan(*ints, plan=far(4096)),
               lambda: binding.dybit_cache_read(calls.cache, calls.plan, k=far(3, 2, 64), v=calls.tensor(3, 2, 64), stream=0),
               lambda: binding.dybit_cache_write(calls.cache, calls.tensor(3, 2, 64), far(3, 2, 64), calls.plan, stream=0)]
    for call in refused:
        with pytest.raises(ValueError):
            call()
    calls.plan.device = 1                                  # a plan of one device, a cache of another
    with pytest.raises(ValueError):
        calls.write()


def test_another_device_than_the_current_one_is_refused(current_device):
    calls, ints = Calls(), [Table(INTS.view(4, 10)), Table(INTS[:5]), Table(INTS[:4])]
    current_device[0] = 1
    for call in (calls.attention, calls.write, lambda: binding.dybit_cache_plan(calls.cache, *ints, 8, 4, stream=0),
                 lambda: binding.dybit_cache_read(calls.cache, calls.plan, k=calls.tensor(3, 2, 64), v=calls.tensor(3, 2, 64), stream=0)):
        with pytest.raises(ValueError):
            call()
