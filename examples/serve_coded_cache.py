"""Serves requests through an attention layer whose weights are 4-bit DyBit codes and whose cache is 8-bit DyBit codes.

The projections are coded products (dybit_gemm); keys and values go into pages of a common pool as they come
(dybit_cache_write), and every step's queries meet the cached codes as they lie (dybit_cache_attention).  A step takes
whatever the requests have: a whole prompt, a piece of one, one token, or none.

    python examples/serve_coded_cache.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2302_12510_b200 as dy  # noqa: E402

W_FMT, X_FMT = (4, True), (8, True)


class CodedAttention:
    """One attention layer: coded projections of queries, keys and values, and of the output."""

    def __init__(self, width, q_heads, heads, dim, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.q_heads, self.heads, self.dim = q_heads, heads, dim
        shapes = ((q_heads + 2 * heads) * dim, width), (width, q_heads * dim)
        self.weights = [(*dy.dybit_quantize_pack_2d(torch.randn(s, generator=g, device=device) / s[1] ** 0.5, W_FMT), s) for s in shapes]

    def project(self, i, x):
        codes_w, scale_w, (N, K) = self.weights[i]
        codes_x, scale_x = dy.dybit_quantize_pack_2d(x, X_FMT)
        return dy.dybit_gemm(x.shape[0], N, K, codes_x, X_FMT, scale_x, codes_w, W_FMT, scale_w)[0]

    def __call__(self, x, cache, plan):
        """x [tokens][width] -> (outputs of the same shape, what the attention got and gave)."""
        qkv = self.project(0, x).bfloat16().view(-1, self.q_heads + 2 * self.heads, self.dim)
        q, k, v = qkv.split([self.q_heads, self.heads, self.heads], dim=1)      # views: the calls take strides
        dy.dybit_cache_write(cache, k, v, plan)
        y = dy.dybit_cache_attention(q, cache, plan)
        return self.project(1, y.flatten(1).float()), (q, k, v, y)


class Pages:
    """Which page of the pool holds which tokens of which request."""

    def __init__(self, cache, requests, most, device="cuda"):
        self.free, self.page = list(range(cache.pages)), cache.page
        self.table = torch.full((requests, most), -1, dtype=torch.int32)
        self.lengths, self.device = [0] * requests, device

    def step(self, cache, new, q_heads):
        """Room for new[b] tokens of request b, and the plan of the step."""
        for b, n in enumerate(new):
            for j in range(-(-self.lengths[b] // self.page), -(-(self.lengths[b] + n) // self.page)):
                self.table[b, j] = self.free.pop()
            self.lengths[b] += n
        starts = torch.tensor([0] + new).cumsum(0)
        ints = lambda t: t.to(torch.int32).to(self.device)
        return dy.CachePlan(cache, ints(self.table), ints(starts), ints(torch.tensor(self.lengths)), sum(new), q_heads, max(new))

    def release(self, b):
        """A request that has ended gives its pages back."""
        self.free += [p for p in self.table[b].tolist() if p >= 0]
        self.table[b], self.lengths[b] = -1, 0


def serve(prompts=(300, 45, 1, 130), steps=8, width=256, q_heads=8, heads=2, dim=64, page=32, seed=0, device="cuda"):
    """Returns, step by step, (new tokens of each request, lengths, queries, keys, values, outputs), the cache and its pages."""
    layer = CodedAttention(width, q_heads, heads, dim, seed, device)
    most = -(-(max(prompts) + steps) // page)
    cache = dy.KVCache(len(prompts) * most, page, heads, dim, device=device)
    pages, record = Pages(cache, len(prompts), most, device), []
    g = torch.Generator(device=device).manual_seed(seed + 1)
    half = prompts[0] // 2
    for i in range(steps):
        # the first prompt comes in two pieces, while the others already go on
        new = [half if i == 0 else prompts[0] - half if i == 1 else 1] + [n if i == 0 else 1 for n in prompts[1:]]
        plan = pages.step(cache, new, q_heads)
        x = torch.randn((sum(new), width), generator=g, device=device)
        _, seen = layer(x, cache, plan)
        record.append((new, list(pages.lengths), *seen))
    return record, cache, pages


def main():
    record, cache, pages = serve()
    held = sum(pages.lengths)
    coded = sum(t.numel() * t.element_size() for t in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales))
    print("%d steps, %d tokens in %d of %d pages" % (len(record), held, cache.pages - len(pages.free), cache.pages))
    print("pool: %.2f MB in codes and scales, %.2f MB as bfloat16" % (coded / 1e6, 4 * cache.k_codes.numel() / 1e6))
    whole = dy.CachePlan(cache, pages.table.to("cuda"), torch.tensor([0] + pages.lengths).cumsum(0).to(torch.int32).to("cuda"),
                         torch.tensor(pages.lengths, dtype=torch.int32, device="cuda"), held)
    k, _ = dy.dybit_cache_read(cache, whole)
    mine = [torch.cat([r[3][sum(r[0][:b]):sum(r[0][:b + 1])] for r in record]) for b in range(len(pages.lengths))]
    k0 = torch.cat(mine).float()
    print("keys in the cache differ from those written by %.2f %%" % (100 * float((k - k0).norm() / k0.norm())))


if __name__ == "__main__":
    main()
