"""The range checks of the fine-tuning operators' debug build: in-range work sets none of them off, whatever its shape, and a
plan that names a token beyond the batch sets one off instead of touching that token.  Run in a child process, since the
library is chosen at import time.  Every buffer is longer than the batch, so the named token is memory of the test's own."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r"""
import torch
import paper_2302_12510_b200 as dy
from paper_2302_12510_b200 import binding, _build
assert binding.lib._name == _build.DEBUG_LIB_PATH, binding.lib._name
dev, g = "cuda:0", torch.Generator().manual_seed(0)
r = lambda *s: torch.randn(s, generator=g)
F, BF = torch.float32, torch.bfloat16

def status():
    torch.cuda.synchronize()
    return dy.dybit_last_device_status()

# shapes: one token, odd sizes, rows that fit registers and rows that do not, several chunks to an adapter, adapters without tokens
for T, K, N, R, n, t in ((1, 64, 64, 8, 1, BF), (17, 1003, 777, 8, 5, F), (130, 200, 136, 32, 3, BF), (1700, 264, 72, 16, 2, F), (90, 72, 264, 128, 40, BF)):
    x, dY = r(T, K).to(dev), r(T, N).to(t).to(dev)
    for xx in (x, x.bfloat16(), x.half()):
        codes, scales = dy.dybit_checkpoint_save(xx, (8, 1))
    for d in (F, BF, torch.float16):
        dy.dybit_checkpoint_load(codes, K, (8, 1), scales, dtype=d)
        dy.dybit_checkpoint_wgrad(dY.to(d), codes, K, (8, 1), scales)
    A, B = r(n, R, K).to(dev).bfloat16(), r(n, R, N).to(dev).bfloat16()
    plan = dy.AdapterPlan(torch.randint(-1, n, (T,), generator=g).to(torch.int32).to(dev), n)
    y, v = dy.dybit_adapters(x.to(t), A, B, None, plan, want_v=True)
    dy.dybit_adapters_backward(dY, codes, (8, 1), scales, A, B, None, plan, v)
    assert status() == (0, 0), (T, K, N, status())
dy.dybit_checkpoint_save(r(3, 20011).to(dev), (8, 1))
dy.dybit_adapters_plan(torch.empty(0, dtype=torch.int32, device=dev), 7)
assert status() == (0, 0)

# a plan that names a token which the batch does not have
T, more, K, N, R, n = 70, 8, 136, 72, 16, 2
whole = dict(x=r(T + more, K).to(dev).bfloat16(), dY=r(T + more, N).to(dev).bfloat16(), y=torch.full((T + more, N), 7.0, device=dev, dtype=BF),
             v=torch.full((T + more, R), 7.0, device=dev), dx=torch.full((T + more, K), 7.0, device=dev, dtype=BF))
codes, scales = dy.dybit_checkpoint_save(whole["x"], (8, 1))
A, B = r(n, R, K).to(dev).bfloat16(), r(n, R, N).to(dev).bfloat16()
ids = (torch.arange(T, dtype=torch.int32) % n).to(dev)
part = {k: w[:T] for k, w in whole.items()}
for place in (0, 5, T - 1):
    plan = dy.AdapterPlan(ids, n)
    plan.buffer.view(torch.int32)[8 + place] = T + 3            # after eight counters: the tokens in their groups' order
    dy.dybit_adapters(part["x"], A, B, None, plan, out=part["y"], v=part["v"])
    st = status()
    assert st[0] == 7 and (st[1] & 3) == 2, st                  # DYBIT_ERR_DEVICE_BOUNDS
    dy.dybit_adapters_backward(part["dY"], codes[:T], (8, 1), scales[:T], A, B, None, plan, part["v"], dx=part["dx"])
    st = status()
    assert st[0] == 7 and (st[1] & 3) == 2, st
    for k in ("y", "v", "dx"):
        assert bool((whole[k][T:] == 7.0).all()), k             # nothing was written there
    assert status() == (0, 0)                                   # read once, cleared
print("range checks ok")
"""


def test_checks_stay_quiet_in_range_and_catch_a_foreign_token():
    from paper_2302_12510_b200 import _build
    if not os.path.exists(_build.DEBUG_LIB_PATH):
        _build.build_library(debug_bounds=True)
    env = dict(os.environ, DYBIT_LIBRARY="debug", PYTHONPATH=ROOT)
    proc = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert proc.returncode == 0, proc.stdout[-2000:] + proc.stderr[-4000:]
    assert "range checks ok" in proc.stdout
