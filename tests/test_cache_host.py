"""CPU-only checks of the key-value cache: sizes, and refusals that are decided before anything is launched."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2302_12510_b200 as dy

L = dy.lib
P = C.c_void_p
OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = range(5)
F32, BF16, F16 = 0, 1, 2


def cache(k=64, v=64, ks=64, vs=64, pages=100, page=64, heads=8, dim=128):
    return dy.binding._CCache(k, v, ks, vs, pages, page, heads, dim)


def batch(sequences=4, tokens=100, max_new=50, q_heads=32, table=64, stride=10, max_pages=10):
    return dy.binding._CCacheBatch(sequences, tokens, max_new, q_heads, table, stride, max_pages, 1, 0)


def plan_bytes(c, b):
    return L.dybit_cache_plan_bytes(C.byref(c), C.byref(b))


def ws_bytes(c, b):
    return L.dybit_cache_attention_workspace_bytes(C.byref(c), C.byref(b))


BAD_CACHES = [(dict(dim=72), UNSUPPORTED), (dict(dim=144), UNSUPPORTED), (dict(dim=0), INVALID), (dict(page=24), UNSUPPORTED), (dict(page=256), UNSUPPORTED),
              (dict(page=0), INVALID), (dict(heads=0), INVALID), (dict(pages=-1), INVALID), (dict(pages=1 << 31), UNSUPPORTED)]
BAD_BATCHES = [(dict(sequences=-1), INVALID), (dict(tokens=-1), INVALID), (dict(q_heads=12), INVALID), (dict(q_heads=0), INVALID), (dict(stride=9), INVALID),
               (dict(max_pages=-1), INVALID), (dict(q_heads=8 * 129), UNSUPPORTED), (dict(tokens=(1 << 26) + 1), UNSUPPORTED),
               (dict(tokens=1 << 26, q_heads=32), UNSUPPORTED), (dict(max_pages=1 << 30, stride=1 << 30), UNSUPPORTED), (dict(sequences=(1 << 20) + 1), UNSUPPORTED)]


@pytest.mark.parametrize("args,status", BAD_CACHES + BAD_BATCHES)
def test_shapes_that_are_refused(args, status):
    mine = {k: v for k, v in args.items() if k in ("dim", "page", "heads", "pages")}
    c, b = cache(**mine), batch(**{k: v for k, v in args.items() if k not in mine})
    launches = dy.dybit_launch_count()
    assert plan_bytes(c, b) == 0 and ws_bytes(c, b) == 0
    rc, rb = C.byref(c), C.byref(b)
    assert L.dybit_cache_plan(rc, rb, P(64), P(64), P(64), 1 << 40, None) == status
    assert L.dybit_cache_write(rc, rb, P(64), P(64), 1024, 128, P(64), 1024, 128, BF16, 2, None) == status
    assert L.dybit_cache_read(rc, rb, P(64), P(64), 1024, 128, P(64), 1024, 128, BF16, None) == status
    assert L.dybit_cache_attention(rc, rb, P(64), P(64), BF16, 4096, 128, P(64), 4096, 128, None, 0.1, 1, 0, P(1024), 1 << 40, None) == status
    assert dy.dybit_launch_count() == launches


def test_plan_arguments():
    c, b = cache(), batch()
    need = plan_bytes(c, b)
    plan = lambda starts=64, lengths=64, at=64, size=need: L.dybit_cache_plan(C.byref(c), C.byref(b), P(starts), P(lengths), P(at), size, None)
    assert plan(starts=0) == INVALID and plan(lengths=0) == INVALID and plan(at=0) == INVALID
    assert plan(starts=66) == ALIGNMENT and plan(at=72) == ALIGNMENT and plan(size=need - 1) == WORKSPACE
    # the memory of the cache is not looked at by a plan
    assert plan_bytes(cache(k=0, v=0, ks=0, vs=0), b) == need


def test_write_and_read_arguments():
    def both(status, write_only=False, c=cache(), b=batch(), plan=64, k=64, kt=1024, kh=128, v=64, vt=1024, vh=128, t=BF16, top=2):
        assert L.dybit_cache_write(C.byref(c), C.byref(b), P(plan), P(k), kt, kh, P(v), vt, vh, t, top, None) == status
        if not write_only:
            assert L.dybit_cache_read(C.byref(c), C.byref(b), P(plan), P(k), kt, kh, P(v), vt, vh, t, None) == status
    for args in (dict(plan=0), dict(k=0), dict(v=0), dict(kt=127), dict(vh=127), dict(t=3), dict(c=cache(k=0)), dict(c=cache(vs=0)), dict(b=batch(table=0))):
        both(INVALID, **args)
    for args in (dict(plan=72), dict(k=65), dict(v=65), dict(t=F32, k=66), dict(c=cache(k=72)), dict(c=cache(ks=66)), dict(b=batch(table=66))):
        both(ALIGNMENT, **args)
    both(INVALID, write_only=True, top=-1)
    both(INVALID, write_only=True, top=7)
    for args in (dict(sequences=0), dict(tokens=0), dict(max_new=0)):
        both(OK, b=batch(**args), k=0, v=0)


def test_attention_arguments():
    c, b = cache(), batch()
    need = ws_bytes(c, b)

    def run(c=c, b=b, plan=64, q=64, t=BF16, qt=4096, qh=128, y=64, yt=4096, yh=128, lse=64, scale=0.1, causal=1, window=0, ws=1024, size=need):
        return L.dybit_cache_attention(C.byref(c), C.byref(b), P(plan), P(q), t, qt, qh, P(y), yt, yh, P(lse), scale, causal, window, P(ws), size, None)
    for args in (dict(plan=0), dict(q=0), dict(y=0), dict(qt=127), dict(yh=127), dict(t=3), dict(window=-1), dict(causal=0, window=3), dict(scale=-1.0),
                 dict(scale=float("nan")), dict(scale=float("inf")), dict(c=cache(v=0)), dict(c=cache(pages=0))):
        assert run(**args) == INVALID, args
    assert run(t=F32) == UNSUPPORTED
    for args in (dict(q=65), dict(y=65), dict(lse=66), dict(ws=1040), dict(plan=72)):
        assert run(**args) == ALIGNMENT, args
    assert run(ws=0) == WORKSPACE and run(size=need - 1) == WORKSPACE
    for args in (dict(sequences=0), dict(tokens=0), dict(max_new=0)):
        assert run(b=batch(**args), q=0, y=0, ws=0, size=0) == OK


def test_sizes_follow_the_batch():
    c = cache()
    one, many = plan_bytes(c, batch(tokens=1, sequences=1, max_new=1)), plan_bytes(c, batch(tokens=8192, sequences=64, max_new=4096))
    assert 0 < one < 1 << 22 and 0 < many < 1 << 22          # (neither is the larger in general: one token has more, smaller tiles)
    # the workspace holds the parts of cut tiles: a size that the number of SMs sets, not the pool or the lengths
    assert ws_bytes(c, batch()) == ws_bytes(cache(pages=1 << 20), batch(max_pages=1 << 20, stride=1 << 20))
    assert ws_bytes(c, batch(tokens=1, max_new=1, sequences=1)) < 64 << 20


def test_binding_checks_its_tensors():
    codes = torch.zeros((4, 2, 16, 64), dtype=torch.uint8)
    with pytest.raises(ValueError):
        dy.KVCache(4, 16, 2, 64, k_codes=codes)


def test_header_documents_every_call():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dybit.h")).read()
    for name in ("dybit_cache_plan", "dybit_cache_write", "dybit_cache_read", "dybit_cache_attention"):
        assert re.search(r"\b%s\(" % name, header) and hasattr(dy, name)
