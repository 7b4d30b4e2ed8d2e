"""The cache's operators together, as the example uses them: prompts in pieces, tokens one by one, pages of a common pool."""
import os
import sys

import pytest
import torch

import paper_2302_12510_b200 as dy

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_outputs_are_the_attention_over_what_the_cache_holds():
    import serve_coded_cache as ex
    steps = 6
    for upto in (1, 2, steps):                             # (a page's scale may still grow: the cache is read as the last step left it)
        record, cache, pages = ex.serve(steps=upto)
        new, lengths, q, k, v, y = record[-1]
        ints = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")
        starts = [sum(lengths[:b]) for b in range(len(lengths) + 1)]
        ks, vs = dy.dybit_cache_read(cache, dy.CachePlan(cache, pages.table.to("cuda"), ints(starts), ints(lengths), sum(lengths)))
        assert sum(lengths) == sum(sum(r[0]) for r in record)
        at, group = 0, q.shape[1] // cache.heads
        for b, n in enumerate(new):
            kb, vb = (t[starts[b]:starts[b + 1]].double().repeat_interleave(group, 1) for t in (ks, vs))
            x = torch.einsum("ihd,jhd->hij", q[at:at + n].double(), kb) * cache.dim ** -0.5
            seen = torch.arange(lengths[b], device="cuda")[None, :] <= lengths[b] - n + torch.arange(n, device="cuda")[:, None]
            w = torch.softmax(x.masked_fill(~seen, -torch.inf), dim=-1)
            want, size = torch.einsum("hij,jhd->ihd", w, vb), torch.einsum("hij,jhd->ihd", w, vb.abs())
            # outputs are rounded to bf16 (2^-8 of themselves at most), probabilities to f16 (2^-11 of what they weigh); scores are below
            # 2^5, so their 64 fp32 sums are off by 64 * 2^-23 * 2^5 * sqrt(64) at most and the outputs by twice that part: below 2^-8
            assert float(x.abs().amax()) < 32.0
            assert bool(((y[at:at + n].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -11) * size + 1e-30).all())
            at += n
        pages.release(1)
        assert len(pages.free) == cache.pages - sum(-(-n // cache.page) for i, n in enumerate(lengths) if i != 1)


def test_example_runs():
    import serve_coded_cache as ex
    ex.main()
