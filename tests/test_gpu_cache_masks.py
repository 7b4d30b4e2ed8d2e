"""Masks of the attention over the cache at the ends of their range, and rows in front of a sequence's first position."""
import pytest
import torch

import paper_2302_12510_b200 as dy
import cache_reference as ref
from test_gpu_cache import BF, DEV, activations, device_cache

pytestmark = pytest.mark.gpu

# with and without rows in front of position 0, in small and in large tiles
BATCHES = [([10, 70, 40], [25, 90, 1]), ([100, 500], [300, 300]), ([0, 3], [5, 2])]


@pytest.mark.parametrize("lengths,news", BATCHES)
def test_windows_that_hold_everything(lengths, news):
    b = ref.Batch(lengths, news, 16, 2, 64, seed=46)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, BF, 3)
    plan = dy.CachePlan(cache, *b.to(DEV), b.T, 8, max(news))
    want = ref.attention(b, q, *pools, 0.125)
    full = dy.dybit_cache_attention(qd, cache, plan, scale=0.125)
    ref.check_attention(full, None, want, BF)
    for window in (1 << 26, (1 << 30) - 1, 2**31 - 50, 2**31 - 2, 2**31 - 1):
        assert torch.equal(dy.dybit_cache_attention(qd, cache, plan, scale=0.125, window=window), full), window
        other = dy.CachePlan(cache, *b.to(DEV), b.T, 8, max(news), window=window)
        assert torch.equal(dy.dybit_cache_attention(qd, cache, other, scale=0.125), full), window


@pytest.mark.parametrize("lengths,news", BATCHES)
def test_rows_in_front_of_the_first_position(lengths, news):
    # they see nothing under a causal mask, with and without a window, and every key without one
    b = ref.Batch(lengths, news, 16, 2, 64, seed=47)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, BF, 3)
    plan = dy.CachePlan(cache, *b.to(DEV), b.T, 8, max(news))
    front = [(i, r) for i in range(len(news)) for r in b.rows(i) if b.position(i, r) < 0]
    assert front
    for causal, window in ((True, 0), (True, 7), (False, 0)):
        lse = torch.empty((b.T, 8), device=DEV)
        y = dy.dybit_cache_attention(qd, cache, plan, scale=0.125, causal=causal, window=window, lse=lse)
        ref.check_attention(y, lse, ref.attention(b, q, *pools, 0.125, causal, window), BF)
        for i, r in front:
            assert bool((y[r] == 0).all() and (lse[r] == -torch.inf).all()) == (causal or lengths[i] == 0)
