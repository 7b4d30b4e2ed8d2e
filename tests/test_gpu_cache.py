"""The key-value cache in 8-bit codes on the GPU, against the definitions in 64 bits: writes and reads bit for bit, attention
within the bound that tests/cache_reference.py derives."""
import math

import pytest
import torch

import paper_2302_12510_b200 as dy
import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, H, F = torch.bfloat16, torch.float16, torch.float32


def device_cache(b, k_pool, v_pool):
    return dy.KVCache(b.pages, b.page, b.heads, b.dim, k_codes=k_pool[0].to(DEV), v_codes=v_pool[0].to(DEV), k_scales=k_pool[1].to(DEV),
                      v_scales=v_pool[1].to(DEV))


def plan_of(cache, b, q_heads=None, max_new=None):
    return dy.CachePlan(cache, *b.to(DEV), b.T, q_heads, max_new)


def activations(b, heads, dtype, seed, packed=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((b.T, heads, b.dim), generator=g) * torch.exp(0.7 * torch.randn((b.T, 1, 1), generator=g))
    x = x.to(dtype)
    if not packed:
        return x, x.to(DEV)
    wide = torch.zeros((b.T, heads + 3, b.dim), dtype=dtype, device=DEV)
    wide[:, 2:2 + heads] = x.to(DEV)
    return x, wide[:, 2:2 + heads]


# lengths, new tokens of each sequence
SHAPES = {
    "one token": ([1], [1]),
    "decode": ([17, 1, 200, 64, 65, 128], [1] * 6),
    "prompts": ([100, 33, 1], [100, 33, 1]),
    "mixed": ([300, 5, 77, 129], [150, 1, 0, 129]),
    "empty": ([0, 40, 0], [0, 3, 2]),
    "longer than there": ([10, 70], [25, 90]),
}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,page,heads,dim", [(BF, 16, 3, 128), (H, 64, 2, 80), (F, 32, 1, 64), (F, 128, 2, 128), (BF, 128, 1, 16)])
def test_write_and_read(shape, dtype, page, heads, dim):
    lengths, news = SHAPES[shape]
    b = ref.Batch(lengths, news, page, heads, dim, seed=len(shape) + page, gap=2)
    pools = [b.pool(2.0), b.pool(2.0)]
    cache = device_cache(b, *pools)
    plan = plan_of(cache, b, max_new=max(max(news), 1))
    (k, kd), (v, vd) = activations(b, heads, dtype, 1, packed=page == 64), activations(b, heads, dtype, 2)
    dy.dybit_cache_write(cache, kd, vd, plan, top=3)
    for x, pool, codes, scales in ((k, pools[0], cache.k_codes, cache.k_scales), (v, pools[1], cache.v_codes, cache.v_scales)):
        want_c, want_s = ref.write(b, x, *pool, top=3)
        assert torch.equal(scales.cpu(), want_s)
        assert torch.equal(codes.cpu(), want_c)
    for out in (F, BF, H):
        kr = torch.full((b.T, heads, dim), 7.0, dtype=out, device=DEV)
        got, _ = dy.dybit_cache_read(cache, plan, dtype=out, k=kr)
        want, mine = ref.read(b, cache.k_codes.cpu(), cache.k_scales.cpu())
        assert torch.equal(got.cpu()[mine], want[mine].to(out))
        assert bool((got.cpu()[~mine] == 7.0).all())          # rows of no sequence


@pytest.mark.parametrize("top", [0, 2, 6])
def test_token_by_token(top):
    # writes of one token each: scales grow, older codes move with them
    page, heads, dim, n = 16, 2, 32, 40
    g = torch.Generator().manual_seed(top)
    x = torch.randn((n, heads, dim), generator=g) * torch.exp2(torch.arange(n) % 16 - 4.0)[:, None, None]
    x[3] = 0.0
    b = ref.Batch([n], [1], page, heads, dim, seed=3)
    cache = dy.KVCache(b.pages, page, heads, dim)
    cache.k_codes.fill_(0x55), cache.v_codes.fill_(0x55)
    codes, scales = cache.k_codes.cpu(), cache.k_scales.cpu()
    for i in range(n):
        b.lengths, b.T = [i + 1], 1
        dy.dybit_cache_write(cache, x[i:i + 1].to(DEV), -x[i:i + 1].to(DEV), plan_of(cache, b), top=top)
        codes, scales = ref.write(b, x[i:i + 1], codes, scales, top)
    assert torch.equal(cache.k_codes.cpu(), codes) and torch.equal(cache.k_scales.cpu(), scales) and torch.equal(cache.v_scales.cpu(), scales)
    whole = ref.Batch([n], [n], page, heads, dim, seed=3)
    back, mirror = dy.dybit_cache_read(cache, plan_of(cache, whole))
    assert torch.equal(back, -mirror)
    # every rounding moves an element by half a step at most: once when it is written, once more whenever its page's scale grows
    room, held = torch.zeros((n, heads, dim), dtype=torch.float64), torch.zeros((-(-n // page), heads), dtype=torch.float64)
    for i in range(n):
        j, first = i // page, i // page * page
        need = torch.tensor([ref.needed_scale(x[i, h].double(), top) for h in range(heads)], dtype=torch.float64)
        new = torch.maximum(held[j], need) if i > first else need
        for h in range(heads):
            if new[h] > 0:
                for r in range(first if new[h] > held[j, h] else i, i + 1):
                    room[r, h] += ref.half_step(x[r, h].double() / new[h] * 1.25) * new[h]
        held[j] = new
    assert bool(((back.cpu().double() - x.double()).abs() <= room).all())


def test_numbers_that_are_not_finite():
    b = ref.Batch([20], [20], 16, 2, 16, seed=5)
    x = torch.randn((20, 2, 16), generator=torch.Generator().manual_seed(1))
    x[2, 0, 3], x[3, 0, 4], x[4, 1, 5] = math.inf, -math.inf, math.nan
    x[16:, 1] = math.nan                                     # a block without a finite number
    x[16:, 0] = math.inf
    for dtype in (F, BF, H):
        cache = dy.KVCache(b.pages, 16, 2, 16)
        codes, scales = cache.k_codes.cpu(), cache.k_scales.cpu()
        dy.dybit_cache_write(cache, x.to(dtype).to(DEV), x.to(dtype).to(DEV), plan_of(cache, b))
        codes, scales = ref.write(b, x.to(dtype), codes, scales, 2)
        touched = b.table[0].long()
        assert torch.equal(cache.v_scales.cpu()[touched], scales[touched])
        got, _ = dy.dybit_cache_read(cache, plan_of(cache, b))
        want, mine = ref.read(b, codes, scales)
        assert torch.equal(got.cpu()[mine].double(), want[mine])
        assert bool(torch.isfinite(got).all())


def test_pages_that_are_not_there():
    b = ref.Batch([100, 90], [100, 90], 16, 2, 64, seed=6)
    for bad in (-1, b.pages, 2**31 - 1, -2**31):
        b.table[0, 2] = bad
        pools = [b.pool(), b.pool()]
        cache = device_cache(b, *pools)
        (k, kd), (v, vd) = activations(b, 2, BF, 1), activations(b, 2, BF, 2)
        plan = plan_of(cache, b, q_heads=4)
        dy.dybit_cache_write(cache, kd, vd, plan)
        want_c, want_s = ref.write(b, k, *pools[0], top=2)
        assert torch.equal(cache.k_codes.cpu(), want_c) and torch.equal(cache.k_scales.cpu(), want_s)
        got, _ = dy.dybit_cache_read(cache, plan)
        assert bool((got[32:48] == 0).all()) and bool((got[48:64] != 0).any())
        q, qd = activations(b, 4, BF, 3)
        y = dy.dybit_cache_attention(qd, cache, plan)
        host = [(cache.k_codes.cpu(), cache.k_scales.cpu()), (cache.v_codes.cpu(), cache.v_scales.cpu())]
        ref.check_attention(y, None, ref.attention(b, q, *host, 64 ** -0.5), BF)


def attention_case(b, group, dtype, causal=True, window=0, scale=None, spread=1.0, seed=9, gain=1.0, max_new=None, packed=False):
    pools = [b.pool(spread), b.pool(spread)]
    cache = device_cache(b, *pools)
    Hq = b.heads * group
    q, qd = activations(b, Hq, dtype, seed, packed)
    if gain != 1.0:
        q, qd = (q * gain).to(dtype), (qd * gain).to(dtype)
    plan = plan_of(cache, b, Hq, max_new or max(max(b.news), 1))
    out = torch.full((b.T, Hq, b.dim), 5.0, dtype=dtype, device=DEV)
    lse = torch.full((b.T, Hq), 5.0, device=DEV)
    scale = b.dim ** -0.5 if scale is None else scale
    y = dy.dybit_cache_attention(qd, cache, plan, scale=scale, causal=causal, window=window, out=out, lse=lse)
    assert y is out
    want = ref.attention(b, q, *pools, scale, causal, window)
    ref.check_attention(y, lse, want, dtype)
    rest = ~want[3]
    assert bool((y.cpu()[rest] == 5.0).all()) and bool((lse.cpu()[rest] == 5.0).all())
    assert dy.dybit_last_device_status() == (0, 0)
    return y


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,page,heads,dim,group", [(BF, 16, 2, 128, 4), (H, 64, 1, 80, 7), (BF, 32, 3, 64, 1), (H, 128, 2, 128, 8), (BF, 64, 1, 16, 3),
                                                        (H, 16, 2, 48, 2)])
def test_attention(shape, dtype, page, heads, dim, group):
    lengths, news = SHAPES[shape]
    attention_case(ref.Batch(lengths, news, page, heads, dim, seed=page + dim, gap=3), group, dtype)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 10000])
@pytest.mark.parametrize("dtype,page,dim,group", [(BF, 16, 64, 4), (H, 64, 128, 5)])
def test_windows(window, dtype, page, dim, group):
    attention_case(ref.Batch([333, 20, 129], [140, 1, 2], page, 1, dim, seed=window), group, dtype, window=window)


@pytest.mark.parametrize("dtype,page,dim,group", [(BF, 16, 64, 4), (H, 32, 96, 1), (BF, 128, 128, 2)])
def test_without_a_causal_mask(dtype, page, dim, group):
    attention_case(ref.Batch([197, 13, 400], [13, 13, 100], page, 2, dim, seed=4), group, dtype, causal=False)
    attention_case(ref.Batch([5], [9], page, 2, dim, seed=4), group, dtype, causal=False)


@pytest.mark.parametrize("dtype", [BF, H])
def test_values_of_very_different_scales(dtype):
    # neighbouring pages 2^+-8 apart (f16 holds no more), so that maxima and exponents move from page to page; sharp rows too
    b = ref.Batch([700, 64], [3, 64], 16, 2, 64, seed=8)
    attention_case(b, 4, dtype, spread=7.0, gain=0.02)
    attention_case(ref.Batch([700], [3], 16, 2, 64, seed=8), 4, dtype, spread=2.0, gain=6.0)


def test_blocks_of_zeros():
    b = ref.Batch([200], [2], 16, 1, 64, seed=11)
    pools = [b.pool(), b.pool()]
    for codes, scales in pools:
        scales[b.table[0, 3].long()] = 0.0
        scales[b.table[0, 0].long()] = 0.0
    cache = device_cache(b, *pools)
    q, qd = activations(b, 4, BF, 3)
    y = dy.dybit_cache_attention(qd, cache, plan_of(cache, b, 4), scale=0.1)
    ref.check_attention(y, None, ref.attention(b, q, *pools, 0.1), BF)


def test_pages_never_written_are_not_looked_at():
    # memory behind a sequence's last token holds anything: codes of other sequences, scales that are not finite
    b = ref.Batch([40, 17], [2, 1], 16, 2, 64, seed=12, spare=6)
    pools = [b.pool(), b.pool()]
    used = torch.cat([b.table[i, :-(-n // 16)] for i, n in enumerate(b.lengths)]).long()
    for codes, scales in pools:
        mask = torch.ones(b.pages, dtype=torch.bool)
        mask[used] = False
        scales[mask] = math.nan
    b.table[1, 2] = int(torch.nonzero(mask)[0])
    cache = device_cache(b, *pools)
    q, qd = activations(b, 4, H, 3)
    y = dy.dybit_cache_attention(qd, cache, plan_of(cache, b, 4))
    ref.check_attention(y, None, ref.attention(b, q, *pools, 64 ** -0.5), H)


def test_rows_that_are_not_finite_keep_to_themselves():
    b = ref.Batch([50, 90], [3, 1], 16, 2, 64, seed=13)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, BF, 3)
    plan = plan_of(cache, b, 8)
    clean = dy.dybit_cache_attention(qd, cache, plan)
    for bad in (math.inf, -math.inf, math.nan):
        p = qd.clone()
        p[1, 5, 7] = bad
        y = dy.dybit_cache_attention(p, cache, plan)
        assert bool(torch.isnan(y[1, 5]).all())
        y[1, 5] = clean[1, 5]
        assert torch.equal(y, clean)


def test_long_sequences_are_cut_and_joined():
    # one sequence, so the keys are cut into many parts; and 200 of them, which are not cut
    for lengths, heads, group, page in (([9000], 1, 4, 64), ([5000, 300], 2, 1, 16), ([260 + 7 * i for i in range(40)], 8, 2, 32)):
        attention_case(ref.Batch(lengths, [1] * len(lengths), page, heads, 64, seed=14), group, BF)
    attention_case(ref.Batch([9000], [5], 64, 1, 128, seed=15), 7, H, window=3000)


def test_equal_calls_give_equal_bits_and_streams_do_not_matter():
    b = ref.Batch([3000, 500, 64], [1, 7, 64], 64, 2, 128, seed=16)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, BF, 3)
    plan = plan_of(cache, b, 8)
    first = dy.dybit_cache_attention(qd, cache, plan)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(3)]
    got = [dy.dybit_cache_attention(qd, cache, plan, stream=s) for s in sides for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(first, y) for y in got)


def test_captured_step_follows_its_inputs():
    # a decode step in a graph: plan, write and attention, replayed with other lengths, tables and tokens
    page, heads, dim, group = 16, 2, 64, 4
    b = ref.Batch([30, 100], [1, 1], page, heads, dim, seed=17, max_pages=16, spare=20)
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    table, starts, lengths = b.to(DEV)
    q, k, v = (torch.zeros((2, n, dim), dtype=BF, device=DEV) for n in (heads * group, heads, heads))
    buffer = torch.empty(dy.dybit_cache_plan_bytes(cache, table, 2, heads * group), dtype=torch.uint8, device=DEV)

    def step():
        plan = dy.CachePlan(cache, table, starts, lengths, 2, heads * group, buffer=buffer)
        dy.dybit_cache_write(cache, k, v, plan)
        return dy.dybit_cache_attention(q, cache, plan), plan

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, keep = step()
    host = [[c.clone() for c in p] for p in pools]
    cache.k_codes.copy_(pools[0][0]), cache.v_codes.copy_(pools[1][0]), cache.k_scales.copy_(pools[0][1]), cache.v_scales.copy_(pools[1][1])
    free = [p for p in range(b.pages) if p not in set(b.table.flatten().tolist())]
    for i in range(5):
        for s in range(2):
            need = -(-b.lengths[s] // page)
            if b.table[s, need - 1] < 0:
                b.table[s, need - 1] = free.pop()
        table.copy_(b.table), lengths.copy_(torch.tensor(b.lengths, dtype=torch.int32))
        new = [torch.randn(t.shape, generator=b.g).to(BF) for t in (q, k, v)]
        for t, x in zip((q, k, v), new):
            t.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        host = [list(ref.write(b, x, *p, top=2)) for x, p in zip(new[1:], host)]
        assert torch.equal(cache.k_codes.cpu(), host[0][0]) and torch.equal(cache.v_scales.cpu(), host[1][1])
        ref.check_attention(y, None, ref.attention(b, new[0], *host, dim ** -0.5), BF)
        b.lengths = [n + 9 if i == 2 else n + 1 for n in b.lengths]


def test_write_then_read_what_attention_sees():
    # the three operators as they are used: prompts are written, then tokens one by one; attention of the same keys and
    # values in plain form agrees with what is read back
    page, heads, dim, group, steps = 32, 2, 128, 4, 6
    b = ref.Batch([70 + steps, 33 + steps], [70, 33], page, heads, dim, seed=18)
    cache = dy.KVCache(b.pages, page, heads, dim)
    for i in range(steps):
        b.news = [70, 33] if i == 0 else [1, 1]
        b.lengths = [70 + i, 33 + i]
        b.starts, b.T = [0, b.news[0], sum(b.news)], sum(b.news)
        (k, kd), (v, vd), (q, qd) = activations(b, heads, BF, 3 * i), activations(b, heads, BF, 3 * i + 1), activations(b, heads * group, BF, 3 * i + 2)
        plan = plan_of(cache, b, heads * group)
        dy.dybit_cache_write(cache, kd, vd, plan)
        y = dy.dybit_cache_attention(qd, cache, plan)
        host = [(cache.k_codes.cpu(), cache.k_scales.cpu()), (cache.v_codes.cpu(), cache.v_scales.cpu())]
        ref.check_attention(y, None, ref.attention(b, q, *host, dim ** -0.5), BF)
        got, _ = dy.dybit_cache_read(cache, plan)
        err = (got.double().cpu() - k.double()).norm() / k.double().norm()
        assert float(err) < 0.05, float(err)


def test_strided_queries_and_outputs():
    b = ref.Batch([100, 40], [10, 1], 16, 2, 64, seed=19)
    attention_case(b, 4, BF, packed=True)
    # rows that start anywhere
    pools = [b.pool(), b.pool()]
    cache = device_cache(b, *pools)
    q, qd = activations(b, 8, BF, 3)
    plan = plan_of(cache, b, 8)
    want = dy.dybit_cache_attention(qd, cache, plan)
    odd = torch.zeros((b.T, 8, 67), dtype=BF, device=DEV)[:, :, 1:65]
    odd.copy_(qd)
    out = torch.zeros((b.T, 9, 65), dtype=BF, device=DEV)[:, 1:, 1:]
    assert torch.equal(dy.dybit_cache_attention(odd, cache, plan, out=out), want)
    k = torch.zeros((b.T, 2, 67), dtype=BF, device=DEV)[:, :, 1:65]
    k.copy_(qd[:, :2])
    dy.dybit_cache_write(cache, k, k, plan)
    codes = cache.k_codes.clone()
    dense = qd[:, :2].contiguous()
    dy.dybit_cache_write(cache, dense, dense, plan)
    assert torch.equal(cache.k_codes, codes)
    into = torch.zeros((b.T, 2, 67), dtype=BF, device=DEV)[:, :, 1:65]
    a, c = dy.dybit_cache_read(cache, plan, dtype=BF, k=into)
    assert torch.equal(a, c)


def test_refusals():
    b = ref.Batch([20], [4], 16, 2, 64, seed=20)
    cache = dy.KVCache(b.pages, 16, 2, 64)
    plan = plan_of(cache, b, 8)
    q, k = torch.zeros((4, 8, 64), dtype=BF, device=DEV), torch.zeros((4, 2, 64), dtype=BF, device=DEV)
    for call in (lambda: dy.dybit_cache_attention(q.float(), cache, plan), lambda: dy.dybit_cache_attention(q[:, :4], cache, plan),
                 lambda: dy.dybit_cache_attention(q[:3], cache, plan), lambda: dy.dybit_cache_attention(q.cpu(), cache, plan),
                 lambda: dy.dybit_cache_attention(q, cache, plan, out=q.half()), lambda: dy.dybit_cache_write(cache, k, k.float(), plan),
                 lambda: dy.dybit_cache_write(cache, k[:, :1], k, plan), lambda: dy.dybit_cache_write(cache, k[:, :1].expand(4, 2, 64), k, plan),
                 lambda: dy.dybit_cache_read(cache, plan, dtype=torch.float64), lambda: dy.dybit_cache_attention(q, dy.KVCache(4, 32, 2, 64), plan),
                 lambda: dy.dybit_cache_attention(q, cache, plan, lse=torch.zeros((4, 8), dtype=BF, device=DEV)),
                 lambda: dy.KVCache(4, 16, 2, 64, k_codes=torch.zeros((4, 2, 16, 32), dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: dy.dybit_cache_attention(q, cache, plan, causal=False, window=4), lambda: dy.dybit_cache_attention(q, cache, plan, window=-1),
                 lambda: dy.dybit_cache_attention(q, cache, plan, ws=torch.empty(1024, dtype=torch.uint8, device=DEV)),
                 lambda: dy.dybit_cache_write(cache, k, k, plan, top=7), lambda: dy.dybit_cache_attention(q, cache, plan, scale=-1.0),
                 lambda: plan_of(dy.KVCache(b.pages, 16, 2, 72), b), lambda: plan_of(dy.KVCache(b.pages, 24, 2, 64), b), lambda: plan_of(cache, b, 3)):
        with pytest.raises(dy.DybitError):
            call()
