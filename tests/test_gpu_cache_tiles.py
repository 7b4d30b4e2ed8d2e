"""The key-value cache's attention where its kernels choose: large and small tiles, work that is cut and joined, masks that the
plan did not expect, maxima that keep rising, pools behind 32-bit offsets.  Bounds: tests/cache_reference.py."""
import pytest
import torch

import paper_2302_12510_b200 as dy
import cache_reference as ref
from test_gpu_cache import BF, DEV, H, activations, attention_case, device_cache, plan_of

pytestmark = pytest.mark.gpu


# many rows of a sequence go to tiles of 256; rows that do not fill one, heads that do not divide one, every width of a head
@pytest.mark.parametrize("lengths,news", [([700, 130], [300, 129]), ([1500], [257]), ([90, 2000, 65], [90, 70, 65]), ([128, 64, 256], [128, 64, 256])])
@pytest.mark.parametrize("dtype,page,heads,dim,group", [(BF, 16, 2, 128, 3), (H, 128, 1, 16, 20), (BF, 64, 2, 48, 5), (H, 32, 3, 80, 7), (BF, 128, 2, 96, 4),
                                                        (H, 64, 4, 64, 8), (BF, 64, 1, 112, 128)])
def test_large_tiles(lengths, news, dtype, page, heads, dim, group):
    attention_case(ref.Batch(lengths, news, page, heads, dim, seed=page + dim + group, gap=1), group, dtype, spread=1.0)


# the sizes around which a batch's rows go to the one or the other kind of tile
@pytest.mark.parametrize("group,news", [(4, [8, 8, 9]), (4, [16, 17]), (1, [33, 32, 31, 64, 65]), (32, [1, 2, 3]), (128, [1, 1]), (7, [1, 4, 5, 10])])
def test_around_the_choice_of_tiles(group, news):
    lengths = [n + 150 * i for i, n in enumerate(news)]
    attention_case(ref.Batch(lengths, news, 32, 2, 64, seed=group), group, BF)
    # the same rows in a batch with many more of them
    attention_case(ref.Batch(lengths + [600], news + [600], 32, 2, 64, seed=group), group, BF)


@pytest.mark.parametrize("group,heads,dim", [(128, 1, 64), (40, 2, 32)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 20), (False, 0)])
def test_large_batches_of_large_groups_have_no_small_tiles(group, heads, dim, causal, window):
    news = [1, 0, 1, 2] * 8
    attention_case(ref.Batch([(37 * i) % 190 + (i > 0) for i in range(32)], news, 16, heads, dim, seed=group, gap=2), group, BF, causal=causal, window=window)


@pytest.mark.parametrize("window", [1, 63, 64, 65, 127, 128, 500])
@pytest.mark.parametrize("dtype,page,dim,group", [(BF, 16, 128, 3), (H, 128, 64, 4)])
def test_windows_of_large_tiles(window, dtype, page, dim, group):
    attention_case(ref.Batch([900, 300], [520, 300], page, 1, dim, seed=window), group, dtype, window=window)


# what the plan expects, what the call asks for
MASKS = [(True, 0), (True, 1), (True, 70), (True, 2000), (False, 0)]


@pytest.mark.parametrize("expects", MASKS)
@pytest.mark.parametrize("news", [[1, 1, 1], [300, 1, 40]])
def test_masks_that_the_plan_does_not_expect(expects, news):
    b = ref.Batch([1300, 20, 400], news, 64, 2, 64, seed=30)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, BF, 3)
    plan = dy.CachePlan(cache, *b.to(DEV), b.T, 8, max(news), causal=expects[0], window=expects[1])
    for causal, window in MASKS:
        y = dy.dybit_cache_attention(qd, cache, plan, causal=causal, window=window)
        ref.check_attention(y, None, ref.attention(b, q, *pools, 64 ** -0.5, causal, window), BF, (causal, window))
    assert dy.dybit_last_device_status() == (0, 0)


@pytest.mark.parametrize("news,group", [([1], 4), ([3], 4), ([200], 4)])
@pytest.mark.parametrize("up", [True, False])
def test_maxima_that_keep_rising(news, group, up):
    # keys whose scale doubles every 48 tokens (or halves): a row's largest score is always in its last (first) block
    page, dim, n = 16, 64, 400
    b = ref.Batch([n], news, page, 2, dim, seed=31)
    pools = [b.pool(), b.pool()]
    k_codes, k_scales = pools[0]
    k_codes.fill_(40), k_codes[..., ::7].fill_(0x80 | 9)
    for j in range(-(-n // page)):
        k_scales[b.table[0, j].long()] = 2.0 ** ((j if up else n // page - j) // 3 - 5)
    cache = device_cache(b, *pools)
    q, _ = activations(b, 2 * group, BF, 3)
    for sign in (1.0, -1.0):                               # scores up to some tens, of either sign
        mine = (q.abs() * sign * torch.where(torch.arange(dim) % 7 == 0, -1.0, 1.0)).to(BF)
        lse = torch.empty((b.T, 2 * group), device=DEV)
        y = dy.dybit_cache_attention(mine.to(DEV), cache, plan_of(cache, b, 2 * group), lse=lse)
        ref.check_attention(y, lse, ref.attention(b, mine, *pools, dim ** -0.5), BF)


def test_large_tiles_with_rows_that_start_anywhere():
    b = ref.Batch([500, 90], [300, 90], 16, 2, 48, seed=32)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, H, 3)
    plan = plan_of(cache, b, 8)
    want = dy.dybit_cache_attention(qd, cache, plan)
    ref.check_attention(want, None, ref.attention(b, q, *pools, 48 ** -0.5), H)
    odd = torch.zeros((b.T, 8, 51), dtype=H, device=DEV)[:, :, 1:49]
    odd.copy_(qd)
    out = torch.zeros((b.T, 9, 49), dtype=H, device=DEV)
    assert torch.equal(dy.dybit_cache_attention(odd, cache, plan, out=out[:, 1:, 1:]), want)
    assert bool((out[:, 0] == 0).all()) and bool((out[:, :, 0] == 0).all())
    heads_first = torch.zeros((8, b.T, 48), dtype=H, device=DEV)
    heads_first.copy_(qd.transpose(0, 1))
    assert torch.equal(dy.dybit_cache_attention(heads_first.transpose(0, 1), cache, plan), want)


def test_pools_behind_32_bit_offsets():
    # the same pages at the front of a small pool and at the end of one of more than 2^32 bytes
    page, heads, dim, group = 128, 8, 128, 2
    b = ref.Batch([300, 1000], [1, 200], page, heads, dim, seed=33)
    pools = [b.pool(), b.pool()]
    small = device_cache(b, *pools)
    big = dy.KVCache(2 ** 32 // (heads * page * dim) + b.pages, page, heads, dim, device=DEV)
    at = big.pages - b.pages
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        getattr(big, name)[at:] = getattr(small, name)
    table, starts, lengths = b.to(DEV)
    wide = torch.full((2, 40), -1, dtype=torch.int32, device=DEV)      # rows of a wider table
    wide[:, 5:5 + table.shape[1]] = torch.where(table >= 0, table + at, table)
    (k, kd), (q, qd) = activations(b, heads, BF, 1), activations(b, heads * group, BF, 2)
    got = []
    for cache, tab in ((small, table), (big, wide[:, 5:5 + table.shape[1]])):
        plan = dy.CachePlan(cache, tab, starts, lengths, b.T, heads * group)
        dy.dybit_cache_write(cache, kd, kd, plan)
        got.append((*dy.dybit_cache_read(cache, plan, dtype=BF), dy.dybit_cache_attention(qd, cache, plan)))
    assert all(torch.equal(a, c) for a, c in zip(*got))
    host = [(small.k_codes.cpu(), small.k_scales.cpu()), (small.v_codes.cpu(), small.v_scales.cpu())]
    ref.check_attention(got[1][2], None, ref.attention(b, q, *host, dim ** -0.5), BF)


def test_batches_without_work_leave_everything_as_it_was():
    b = ref.Batch([50], [4], 16, 2, 64, seed=34)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    q, k = torch.zeros((4, 8, 64), dtype=BF, device=DEV), torch.ones((4, 2, 64), dtype=BF, device=DEV)
    none = torch.zeros((0, 3), dtype=torch.int32, device=DEV)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    for table, starts, lengths, tokens in ((none, ints(0), ints(), 4), (b.table.to(DEV), ints(0, 0), ints(50), 4), (b.table.to(DEV), ints(2, 2), ints(0), 4)):
        plan = dy.CachePlan(cache, table, starts, lengths, tokens, 8)
        out, back = torch.full((4, 8, 64), 5.0, dtype=BF, device=DEV), torch.full((4, 2, 64), 5.0, device=DEV)
        dy.dybit_cache_write(cache, k, k, plan)
        dy.dybit_cache_read(cache, plan, k=back, v=back.clone())
        dy.dybit_cache_attention(q, cache, plan, out=out)
        assert bool((out == 5.0).all()) and bool((back == 5.0).all())
        assert torch.equal(cache.k_codes.cpu(), pools[0][0]) and torch.equal(cache.v_scales.cpu(), pools[1][1])
    plan = dy.CachePlan(cache, b.table.to(DEV), ints(0, 4), ints(50), 4, 8, max_new=3)      # one token more than the plan allows
    out = torch.full((4, 8, 64), 5.0, dtype=BF, device=DEV)
    dy.dybit_cache_attention(q, cache, plan, out=out)
    assert bool((out[3] == 5.0).all()) and bool((out[:3] != 5.0).all())
    assert dy.dybit_last_device_status() == (0, 0)


def test_two_graphs_share_a_workspace():
    # two layers' attention, captured apart, replayed one after another in either order
    b = ref.Batch([3000, 600, 200], [1, 1, 100], 64, 2, 64, seed=35)
    plan, layers = None, []
    ws = None
    for i in range(2):
        pools = [b.pool(), b.pool()]
        cache = device_cache(b, *pools)
        q, qd = activations(b, 8, BF, 3 + i)
        plan = plan or plan_of(cache, b, 8)
        ws = ws if ws is not None else torch.empty(dy.dybit_cache_attention_workspace_bytes(cache, plan) + 1024, dtype=torch.uint8, device=DEV)
        off = -ws.data_ptr() % 1024
        out = torch.zeros_like(qd)
        call = lambda qd=qd, cache=cache, out=out: dy.dybit_cache_attention(qd, cache, plan, out=out, ws=ws[off:])
        call()
        want = out.clone()
        ref.check_attention(want, None, ref.attention(b, q, *pools, 64 ** -0.5), BF)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        layers.append((graph, out, want, (cache, qd)))     # a graph holds none of its tensors
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for _, out, _, _ in layers:
            out.zero_()
        for i in order * 5:
            layers[i][0].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, want) for _, out, want, _ in layers)


def test_calls_of_every_kind_side_by_side_on_two_streams():
    # one plan, two layers with caches of their own, each on its stream; then the same one after another
    b = ref.Batch([900, 77, 64], [1, 40, 64], 16, 2, 128, seed=36)
    sides, results = [torch.cuda.Stream(), torch.cuda.Stream()], []
    plan = None
    for streams in (sides, [torch.cuda.current_stream()] * 2):
        mine = []
        for i, s in enumerate(streams):
            g = torch.Generator().manual_seed(i)
            b.g = g
            cache = device_cache(b, b.pool(), b.pool())
            plan = plan or plan_of(cache, b, 8)
            (_, kd), (_, qd) = activations(b, 2, BF, 10 + i), activations(b, 8, BF, 20 + i)
            mine.append((cache, kd, qd))
        torch.cuda.synchronize()
        got = []
        for _ in range(4):
            for (cache, kd, qd), s in zip(mine, streams):
                dy.dybit_cache_write(cache, kd, kd, plan, stream=s)
                got.append(dy.dybit_cache_attention(qd, cache, plan, stream=s))
                got += dy.dybit_cache_read(cache, plan, dtype=BF, stream=s)
        torch.cuda.synchronize()
        results.append(got)
    assert all(torch.equal(a, c) for a, c in zip(*results))
