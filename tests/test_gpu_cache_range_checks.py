"""The range checks of the key-value cache's debug build: work of every kind sets none of them off, and a plan that names rows beyond the
batch sets them off instead of storing there.  Run in a child process, since the library is chosen at import time.  Every buffer
is longer than the batch, so the named rows are memory of the test's own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r"""
import sys
import torch
sys.path.insert(0, "tests")
import cache_reference as ref
import paper_2302_12510_b200 as dy
from paper_2302_12510_b200 import binding, _build
assert binding.lib._name == _build.DEBUG_LIB_PATH, binding.lib._name
dev, BF = "cuda:0", torch.bfloat16

def status():
    torch.cuda.synchronize()
    return dy.dybit_last_device_status()

def setting(lengths, news, page, heads, dim, **more):
    b = ref.Batch(lengths, news, page, heads, dim, seed=50, **more)
    pools = dict(zip(("k_codes", "k_scales", "v_codes", "v_scales"), [x.to(dev) for p in (b.pool(), b.pool()) for x in p]))
    return b, dy.KVCache(b.pages, page, heads, dim, **pools)

# one token, many, parts joined by warps and by blocks, large tiles whole and cut, no work, sequences that are cut
for lengths, news, page, heads, dim, group, max_new in (([1], [1], 16, 1, 16, 1, 1), ([70] * 90, [1] * 90, 32, 2, 64, 4, 1), ([40000], [1], 64, 2, 128, 4, 1),
                                                        ([3000, 9], [5, 2], 16, 3, 80, 7, 5), ([2000, 300], [600, 300], 128, 2, 128, 4, 600),
                                                        ([9000], [130], 64, 1, 48, 8, 130), ([0, 5], [0, 9], 16, 2, 32, 3, 9), ([300], [200], 16, 2, 64, 4, 150)):
    b, cache = setting(lengths, news, page, heads, dim, gap=1)
    x = lambda n: torch.randn((b.T, n, dim), generator=b.g).to(BF).to(dev)
    for window in (0, 100):
        plan = dy.CachePlan(cache, *b.to(dev), b.T, heads * group, max_new, window=window)
        dy.dybit_cache_write(cache, x(heads), x(heads), plan)
        dy.dybit_cache_read(cache, plan)
        lse = torch.empty((b.T, heads * group), device=dev)
        for causal, w in ((True, 0), (True, 100), (False, 0)):
            dy.dybit_cache_attention(x(heads * group), cache, plan, causal=causal, window=w, lse=lse)
            assert status() == (0, 0), (lengths, causal, w, status())

# rows that the batch does not have: items, tiles and blocks' starts name row T + 3
T, more, heads, group, dim = 1, 8, 1, 4, 64
b, cache = setting([40], [1], 16, heads, dim)
q, y, lse = (torch.full((T + more, heads * group) + s, 7.0, dtype=t, device=dev) for s, t in (((dim,), BF), ((dim,), BF), ((), torch.float32)))
k, v = (torch.full((T + more, heads, dim), 7.0, device=dev) for _ in range(2))
plan = dy.CachePlan(cache, *b.to(dev), T, heads * group, 1)
words = plan.buffer[:plan.buffer.numel() // 4 * 4].view(torch.int32)
dy.dybit_cache_attention(q[:T], cache, plan, out=y[:T], lse=lse[:T])
assert status() == (0, 0) and bool((y[:T] != 7.0).any()) and bool((y[T:] == 7.0).all())
# sixteen counts, an item {row, position, count, sequence}, a tile {row, ...} of eight words, blocks' starts of twelve with their tile from the fifth word on
assert words[16:20].tolist() == [0, 39, 1, 0] and words[20:23].tolist() == [0, 1, 40]
blocks = int(words[2])
assert words[3:5].tolist() == [0, 0]                        # nothing is joined
assert all(words[28 + 12 * i + 4:28 + 12 * i + 7].tolist() == [0, 1, 40] for i in range(blocks))
words[16] = T + 3
dy.dybit_cache_read(cache, plan, k=k[:T], v=v[:T])
st = status()
assert st[0] == 7 and (st[1] & 3) == 2, st                  # DYBIT_ERR_DEVICE_BOUNDS
assert bool((k == 7.0).all() and (v == 7.0).all())
y.fill_(7.0), lse.fill_(7.0)
words[20] = T + 3
for i in range(blocks):
    words[28 + 12 * i + 4] = T + 3
dy.dybit_cache_attention(q[:T], cache, plan, out=y[:T], lse=lse[:T])
st = status()
assert st[0] == 7 and (st[1] & 3) == 2, st
assert bool((y == 7.0).all() and (lse == 7.0).all())
print("ok")
"""


def test_range_checks():
    from paper_2302_12510_b200 import _build
    if not os.path.exists(_build.DEBUG_LIB_PATH):
        _build.build_library(debug_bounds=True)
    env = dict(os.environ, DYBIT_LIBRARY="debug", PYTHONPATH=ROOT)
    proc = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0, proc.stdout[-2000:] + proc.stderr[-4000:]
    assert proc.stdout.endswith("ok\n")
