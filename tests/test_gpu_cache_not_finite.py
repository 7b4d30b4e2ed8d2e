"""Rows of queries that are not finite, in every kind of tile: their own outputs are NaN, and no other row notices."""
import math

import pytest
import torch

import paper_2302_12510_b200 as dy
import cache_reference as ref
from test_gpu_cache import BF, DEV, H, activations, device_cache, plan_of

pytestmark = pytest.mark.gpu

BATCHES = [([1, 40, 7], [1, 3, 2]), ([300], [300]), ([5000], [1])]


@pytest.mark.parametrize("lengths,news", BATCHES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype,same_sign", [(BF, True), (H, False), (H, True)])
def test_rows_that_are_not_finite(lengths, news, bad, dtype, same_sign):
    b = ref.Batch(lengths, news, 16, 2, 64, seed=44)
    pools = [b.pool(), b.pool()]
    if same_sign:                                          # every score of the row is an infinity of one sign
        pools[0][0].copy_((pools[0][0] & 0x7f) | 1)
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, dtype, 3)
    plan = plan_of(cache, b, 8)
    lse = [torch.empty((b.T, 8), device=DEV) for _ in range(2)]
    clean = dy.dybit_cache_attention(qd, cache, plan, lse=lse[0])
    p, hit = qd.clone(), [(0, 2, 7), (b.T - 1, 5, 0), (b.T // 2, 7, 63)]
    for t, h, d in hit:
        p[t, h, d] = bad
    y = dy.dybit_cache_attention(p, cache, plan, lse=lse[1])
    for t, h, _ in hit:
        assert bool(torch.isnan(y[t, h]).all()), (t, h)
        assert not math.isfinite(float(lse[1][t, h]))
        y[t, h], lse[1][t, h] = clean[t, h], lse[0][t, h]
    # (a warp raises the maxima of its rows together, so that a row's roundings may depend on its neighbours: the bound holds for both)
    want = ref.attention(b, q, *pools, 0.125)
    ref.check_attention(clean, lse[0], want, dtype)
    ref.check_attention(y, lse[1], want, dtype)
    assert dy.dybit_last_device_status() == (0, 0)
