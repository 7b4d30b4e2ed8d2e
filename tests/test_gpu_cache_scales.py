"""Scales of pages at the ends of what the attention over the cache takes, and of pages that no row sees.  Bounds: tests/cache_reference.py."""
import math

import pytest
import torch

import paper_2302_12510_b200 as dy
import cache_reference as ref
from test_gpu_cache import BF, DEV, activations, device_cache

pytestmark = pytest.mark.gpu

# single tokens and a few (small tiles), many (large ones); one sequence alone has its keys cut into parts
BATCHES = [([333, 129, 2000], [1, 2, 1]), ([900], [520]), ([5000], [1])]


@pytest.mark.parametrize("lengths,news", BATCHES)
@pytest.mark.parametrize("odd", [2.0 ** 120, 2.0 ** -120, math.inf, math.nan, 0.0])
@pytest.mark.parametrize("window,dim", [(100, 64), (70, 128), (37, 64), (21, 128)])
def test_pages_in_front_of_the_window_are_not_looked_at(lengths, news, odd, window, dim):
    # a page that its sequence has slid past may be another's by now, or hold anything; the keys that a row sees begin inside a tile's unit
    b = ref.Batch(lengths, news, 16, 2, dim, seed=41)
    pools, stale = [b.pool(2.0), b.pool(2.0)], []
    for codes, scales in pools:
        s = scales.clone()
        for i, n in enumerate(lengths):
            gone = max(0, n - news[i] + 1 - window) // 16
            s[b.table[i, :gone].long()] = odd
        stale.append((codes, s))
    cache = device_cache(b, *stale)
    q, qd = activations(b, 8, BF, 3)
    want = ref.attention(b, q, *pools, dim ** -0.5, True, window)
    for expects in (0, window):
        plan = dy.CachePlan(cache, *b.to(DEV), b.T, 8, max(news), window=expects)
        lse = torch.empty((b.T, 8), device=DEV)
        ref.check_attention(dy.dybit_cache_attention(qd, cache, plan, window=window, lse=lse), lse, want, BF, (odd, window, expects))


@pytest.mark.parametrize("lengths,news", BATCHES)
@pytest.mark.parametrize("window", [0, 300])
def test_scales_as_far_apart_as_they_may_be(lengths, news, window):
    # values' scales within 2^98 of each other, neighbouring pages anywhere among them
    b = ref.Batch(lengths, news, 16, 2, 64, seed=42)
    pools = [b.pool(1.0), b.pool(49.0)]
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, BF, 3)
    lse = torch.empty((b.T, 8), device=DEV)
    y = dy.dybit_cache_attention(qd, cache, dy.CachePlan(cache, *b.to(DEV), b.T, 8, max(news)), window=window, lse=lse)
    ref.check_attention(y, lse, ref.attention(b, q, *pools, 64 ** -0.5, True, window), BF)


@pytest.mark.parametrize("lengths,news", BATCHES)
def test_blocks_of_zeros_in_every_kind_of_tile(lengths, news):
    b = ref.Batch(lengths, news, 32, 2, 64, seed=43)
    pools = [b.pool(2.0), b.pool(2.0)]
    for codes, scales in pools:
        for i in range(len(lengths)):
            scales[b.table[i, ::3].long()] = 0.0           # the first page among them
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, BF, 3)
    lse = torch.empty((b.T, 8), device=DEV)
    y = dy.dybit_cache_attention(qd, cache, dy.CachePlan(cache, *b.to(DEV), b.T, 8, max(news)), lse=lse)
    ref.check_attention(y, lse, ref.attention(b, q, *pools, 64 ** -0.5), BF)
