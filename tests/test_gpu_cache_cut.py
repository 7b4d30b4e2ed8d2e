"""Sequences that have more than their batch allows, more new tokens than max_new or more tokens than their row of the table has pages
for: what remains of them keeps its positions."""
import pytest
import torch

import paper_2302_12510_b200 as dy
import cache_reference as ref
from test_gpu_cache import BF, DEV, activations, device_cache

pytestmark = pytest.mark.gpu


class CutBatch(ref.Batch):
    """`lengths` and `news` as they are given to the plan; the 64-bit forms see what is left of them: the first new tokens."""

    def __init__(self, lengths, news, page, heads, dim, seed, max_new, max_pages):
        super().__init__([min(n, max_pages * page) for n in lengths], news, page, heads, dim, seed=seed, gap=1, max_pages=max_pages)
        self.given = torch.tensor(lengths, dtype=torch.int32)
        beyond = [max(0, n - max_new, ln - max_pages * page) for n, ln in zip(news, lengths)]
        self.first = [ln - n for ln, n in zip(lengths, news)]
        self.news = [max(0, n - o) for n, o in zip(news, beyond)]
        self.lengths = [max(0, ln - o) for ln, o in zip(lengths, beyond)]

    def rows(self, b):
        return range(self.starts[b], self.starts[b] + self.news[b])

    def position(self, b, row):
        return self.first[b] + row - self.starts[b]

    def to(self, dev):
        table, starts, _ = super().to(dev)
        return table, starts, self.given.to(dev)


CASES = [
    # lengths, new tokens, max_new, pages to a row (of 16)
    ([50, 80, 7], [4, 20, 7], 3, 8),
    ([50, 2, 90], [5, 9, 1], 4, 8),                        # fewer tokens than new rows, and fewer than are left out
    ([700, 130], [300, 129], 250, 48),                     # large tiles
    ([70, 64, 65], [10, 3, 1], 10, 4),                     # longer than the table: the last tokens have no page
    ([70, 90, 3], [4, 40, 3], 40, 4),                      # all or most of the new tokens
    ([400], [300], 290, 20),                               # both
]


@pytest.mark.parametrize("lengths,news,max_new,max_pages", CASES)
def test_what_is_left_keeps_its_positions(lengths, news, max_new, max_pages):
    b = CutBatch(lengths, news, 16, 2, 64, 45, max_new, max_pages)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    plan = dy.CachePlan(cache, *b.to(DEV), b.T, 8, max_new)
    (k, kd), (q, qd) = activations(b, 2, BF, 1), activations(b, 8, BF, 2)
    dy.dybit_cache_write(cache, kd, kd, plan)
    host = [ref.write(b, k, *p, top=2) for p in pools]
    assert torch.equal(cache.k_codes.cpu(), host[0][0]) and torch.equal(cache.k_scales.cpu(), host[0][1])
    assert torch.equal(cache.v_codes.cpu(), host[1][0]) and torch.equal(cache.v_scales.cpu(), host[1][1])
    back = torch.full((b.T, 2, 64), 7.0, device=DEV)
    dy.dybit_cache_read(cache, plan, k=back, v=back.clone())
    want, mine = ref.read(b, *host[0])
    assert torch.equal(back.cpu()[mine], want[mine].float()) and bool((back.cpu()[~mine] == 7.0).all())
    for window in (0, 33):
        y, lse = torch.full((b.T, 8, 64), 5.0, dtype=BF, device=DEV), torch.full((b.T, 8), 5.0, device=DEV)
        dy.dybit_cache_attention(qd, cache, plan, window=window, out=y, lse=lse)
        ref.check_attention(y, lse, ref.attention(b, q, *host, 0.125, True, window), BF)
        assert bool((y.cpu()[~mine] == 5.0).all()) and bool((lse.cpu()[~mine] == 5.0).all())
    assert dy.dybit_last_device_status() == (0, 0)
