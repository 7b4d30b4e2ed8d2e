"""Batches at the ends of their sizes: none at all, and more sequences and tiles than the plan's block takes at a time."""
import pytest
import torch

import paper_2302_12510_b200 as dy
import cache_reference as ref
from test_gpu_cache import BF, DEV, H, activations, attention_case, device_cache

pytestmark = pytest.mark.gpu


# sequences beyond 1024 (threads of the plan) and 2048 (tiles that it searches in shared memory), tiles of 8, 16 and 256 rows
@pytest.mark.parametrize("sequences,most,group,heads,window", [(1025, 1, 4, 1, 0), (2500, 1, 2, 1, 0), (2100, 3, 4, 1, 20), (1100, 40, 2, 1, 0)])
def test_many_sequences(sequences, most, group, heads, window):
    g = torch.Generator().manual_seed(sequences)
    news = torch.randint(0, most + 1, (sequences,), generator=g).tolist()
    lengths = [n + int(x) for n, x in zip(news, torch.randint(0, 100, (sequences,), generator=g))]
    attention_case(ref.Batch(lengths, news, 32, heads, 32, seed=sequences, gap=1), group, H if most == 1 else BF, window=window)


def test_writes_and_reads_of_many_sequences():
    n = 1500
    b = ref.Batch([1 + i % 37 for i in range(n)], [min(1 + i % 37, 1 + i % 5) for i in range(n)], 16, 1, 16, seed=51)
    pools = [b.pool(2.0), b.pool(2.0)]
    cache = device_cache(b, *pools)
    plan = dy.CachePlan(cache, *b.to(DEV), b.T, max_new=5)
    k, kd = activations(b, 1, BF, 1)
    dy.dybit_cache_write(cache, kd, kd, plan)
    want = ref.write(b, k, *pools[0], top=2)
    assert torch.equal(cache.k_codes.cpu(), want[0]) and torch.equal(cache.k_scales.cpu(), want[1])
    back, _ = dy.dybit_cache_read(cache, plan)
    assert torch.equal(back.cpu(), ref.read(b, *want)[0].float())


def test_a_batch_without_tokens():
    b = ref.Batch([5, 9], [0, 0], 16, 2, 64, seed=52)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    plan = dy.CachePlan(cache, *b.to(DEV), 0, 8)
    none = torch.zeros((0, 2, 64), dtype=BF, device=DEV)
    dy.dybit_cache_write(cache, none, none, plan)
    k, v = dy.dybit_cache_read(cache, plan, dtype=BF)
    y = dy.dybit_cache_attention(torch.zeros((0, 8, 64), dtype=BF, device=DEV), cache, plan)
    assert k.shape == v.shape == (0, 2, 64) and y.shape == (0, 8, 64)
    assert torch.equal(cache.k_codes.cpu(), pools[0][0]) and torch.equal(cache.v_scales.cpu(), pools[1][1])
    assert dy.dybit_last_device_status() == (0, 0)


def test_a_ring_of_pages_serves_a_window():
    # a sequence that slides over a few pages: what lies in front of the window has been written over, and its entries name the same pages
    page, heads, dim, window, ring = 16, 2, 64, 40, 5
    b = ref.Batch([400], [1], page, heads, dim, seed=53)
    cache = dy.KVCache(ring, page, heads, dim)
    g = torch.Generator().manual_seed(1)
    x = torch.randn((400, heads, dim), generator=g) * torch.exp2(torch.arange(400) // 30 * 8.0 - 48)[:, None, None]
    table = (torch.arange(b.most, dtype=torch.int32) % ring).view(1, -1)
    at = 0
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    for n in (7, 33, 1, 1, 30, 9, 40, 1, 25, 1, 39, 40, 40, 40, 33, 30, 29, 1):
        # what the step's tokens may need has to be in the ring with them
        if n + window > ring * page - page:
            n = ring * page - page - window
        plan = dy.CachePlan(cache, table.to(DEV), ints(0, n), ints(at + n), n, 8, window=window)
        kd = x[at:at + n].to(DEV)
        dy.dybit_cache_write(cache, kd, kd, plan)
        at += n
        q = torch.randn((n, 8, dim), generator=g).to(BF) * 0.01
        lse = torch.empty((n, 8), device=DEV)
        y = dy.dybit_cache_attention(q.to(DEV), cache, plan, window=window, lse=lse)
        here = ref.Batch([at], [n], page, heads, dim, seed=0)
        here.pages, here.table, here.starts, here.T = ring, table[:, :-(-at // page)], [0, n], n
        host = [(cache.k_codes.cpu(), cache.k_scales.cpu()), (cache.v_codes.cpu(), cache.v_scales.cpu())]
        ref.check_attention(y, lse, ref.attention(here, q, *host, dim ** -0.5, True, window), BF, (at, n))
