"""The key-value cache on the range-checked debug build: the same results as on the product library, status word clean.  Run in a
child process, since the library is chosen at import time."""
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
assert binding.lib._name == (_build.DEBUG_LIB_PATH if sys.argv[1] == "debug" else _build.LIB_PATH), binding.lib._name
dev, out = "cuda:0", []
for lengths, news, page, heads, dim, group, t in (([40, 700], [1, 1], 16, 2, 64, 4, torch.bfloat16), ([300, 77, 5], [200, 3, 9], 64, 2, 80, 3, torch.float16),
                                                  ([5000], [2], 128, 1, 128, 8, torch.bfloat16)):
    b = ref.Batch(lengths, news, page, heads, dim, seed=page, gap=1)
    cache = dy.KVCache(b.pages, page, heads, dim, **dict(zip(("k_codes", "k_scales", "v_codes", "v_scales"), [x.to(dev) for p in (b.pool(), b.pool()) for x in p])))
    r = lambda n: torch.randn((b.T, n, dim), generator=b.g).to(t).to(dev)
    plan = dy.CachePlan(cache, *b.to(dev), b.T, heads * group)
    dy.dybit_cache_write(cache, r(heads), r(heads), plan)
    lse, into = torch.zeros((b.T, heads * group), device=dev), [torch.zeros((b.T, heads, dim), device=dev) for _ in range(2)]
    for causal, window in ((True, 0), (True, 50), (False, 0)):
        y = torch.zeros((b.T, heads * group, dim), dtype=t, device=dev)
        out += [dy.dybit_cache_attention(r(heads * group), cache, plan, causal=causal, window=window, out=y, lse=lse), lse.clone()]
    dy.dybit_cache_read(cache, plan, k=into[0], v=into[1])
    out += into + [cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales]
torch.cuda.synchronize()
assert dy.dybit_last_device_status() == (0, 0), dy.dybit_last_device_status()
torch.save([o.cpu() for o in out], sys.argv[2])
"""


def test_debug_build_gives_the_same_results(tmp_path):
    import torch
    from paper_2302_12510_b200 import _build
    if not os.path.exists(_build.DEBUG_LIB_PATH):
        _build.build_library(debug_bounds=True)
    results = []
    for name in ("product", "debug"):
        env = dict(os.environ, DYBIT_LIBRARY=name, PYTHONPATH=ROOT)
        path = str(tmp_path / name)
        proc = subprocess.run([sys.executable, "-c", SCRIPT, name, path], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
        assert proc.returncode == 0, proc.stdout[-2000:] + proc.stderr[-4000:]
        results.append(torch.load(path))
    assert all(torch.equal(a, b) for a, b in zip(*results))
