"""The fine-tuning operators on the range-checked debug build: the same results as on the product library, status word
clean.  Run in a child process, since the library is chosen at import time."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r"""
import sys
import torch
import paper_2302_12510_b200 as dy
from paper_2302_12510_b200 import binding, _build
assert binding.lib._name == (_build.DEBUG_LIB_PATH if sys.argv[1] == "debug" else _build.LIB_PATH), binding.lib._name
dev, g = "cuda:0", torch.Generator().manual_seed(0)
r = lambda *s: torch.randn(s, generator=g)
out = []
for T, K, N, R, n, t in ((1, 64, 64, 8, 1, torch.bfloat16), (130, 203, 77, 16, 3, torch.float32), (700, 512, 264, 64, 2, torch.bfloat16)):
    x, dY = r(T, K).to(dev), r(T, N).to(t).to(dev)
    codes, scales = dy.dybit_checkpoint_save(x, (8, 1))
    out += [codes, scales, dy.dybit_checkpoint_load(codes, K, (8, 1), scales), dy.dybit_checkpoint_wgrad(dY, codes, K, (8, 1), scales)]
    A, B = r(n, R, K).to(dev).bfloat16(), r(n, R, N).to(dev).bfloat16()
    plan = dy.AdapterPlan((torch.arange(T, dtype=torch.int32) % (n + 1) - 1).to(dev), n)
    y, v = dy.dybit_adapters(x, A, B, None, plan, want_v=True)
    out += [y, v, *dy.dybit_adapters_backward(dY, codes, (8, 1), scales, A, B, None, plan, v)]
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
