"""Calls of the key-value cache that are refused, and their nearest neighbours that are not."""
import pytest
import torch

import paper_2302_12510_b200 as dy
import cache_reference as ref
from test_gpu_cache import BF, DEV, activations, device_cache

pytestmark = pytest.mark.gpu


def test_a_table_that_is_shared_is_given_as_a_copy():
    # requests that share all their pages: the expanded table is refused, a copy of it is right
    b = ref.Batch([70, 70, 70], [2, 2, 2], 16, 2, 64, seed=40)
    b.table[1:] = b.table[0]
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    table, starts, lengths = b.to(DEV)
    for bad in (table[:1].expand(3, -1), table[0].as_strided((3, table.shape[1]), (1, 1))):
        with pytest.raises(ValueError):
            dy.CachePlan(cache, bad, starts, lengths, b.T, 8)
        with pytest.raises(ValueError):
            dy.dybit_cache_plan_bytes(cache, bad, b.T, 8)
    q, qd = activations(b, 8, BF, 3)
    plan = dy.CachePlan(cache, table[:1].expand(3, -1).contiguous(), starts, lengths, b.T, 8)
    ref.check_attention(dy.dybit_cache_attention(qd, cache, plan), None, ref.attention(b, q, *pools, 64 ** -0.5), BF)
