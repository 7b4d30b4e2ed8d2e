"""CPU-only checks of the fine-tuning operators: sizes, and refusals that are decided before anything is launched."""
import ctypes
import re

import pytest
import torch

import paper_2302_12510_b200 as dy

L = dy.lib
F8, U8, F4 = (dy.binding._CFmt(8, 1), dy.binding._CFmt(8, 0), dy.binding._CFmt(4, 1))
P = ctypes.c_void_p
OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = range(5)
F32, BF16, F16 = 0, 1, 2


def test_save_arguments():
    def save(x=64, t=F32, rows=4, cols=100, ld=100, fmt=F8, top=2, codes=64, stride=128, scales=64):
        return L.dybit_checkpoint_save(P(x), t, rows, cols, ld, fmt, top, P(codes), stride, P(scales), None)
    assert save(fmt=F4) == UNSUPPORTED and save(fmt=dy.binding._CFmt(9, 1)) == INVALID
    assert save(rows=-1) == INVALID and save(ld=99) == INVALID and save(stride=96) == INVALID
    assert save(top=-1) == INVALID and save(top=7) == INVALID and save(fmt=U8, top=8) == INVALID
    assert save(t=3) == INVALID and save(x=0) == INVALID and save(codes=0) == INVALID and save(scales=0) == INVALID
    assert save(stride=136) == ALIGNMENT and save(codes=72) == ALIGNMENT and save(x=66) == ALIGNMENT and save(scales=66) == ALIGNMENT
    assert save(t=BF16, x=65) == ALIGNMENT
    assert save(rows=0) == OK


def test_load_arguments():
    def load(codes=64, stride=128, scales=64, ss=1, rows=4, cols=100, fmt=F8, y=64, t=F32, ld=100):
        return L.dybit_checkpoint_load(P(codes), stride, P(scales), ss, rows, cols, fmt, P(y), t, ld, None)
    assert load(fmt=F4) == UNSUPPORTED and load(ld=99) == INVALID and load(ss=-1) == INVALID and load(t=7) == INVALID
    assert load(y=0) == INVALID and load(scales=0) == INVALID and load(codes=0) == INVALID
    assert load(y=66) == ALIGNMENT and load(codes=65) == ALIGNMENT
    assert load(rows=0) == OK and load(cols=0, ld=0) == OK


def test_wgrad_arguments():
    need = L.dybit_checkpoint_wgrad_workspace_bytes(32, 40, 100, BF16)
    assert need > 0
    for bad in ((-1, 40, 100, BF16), (32, 0, 100, BF16), (32, 40, 0, BF16), (32, 40, 100, 3)):
        assert L.dybit_checkpoint_wgrad_workspace_bytes(*bad) == 0
    # more terms of dY, more room
    assert L.dybit_checkpoint_wgrad_workspace_bytes(320, 400, 100, F32) > L.dybit_checkpoint_wgrad_workspace_bytes(320, 400, 100, F16)

    def wgrad(T=32, N=40, K=100, dY=64, t=BF16, ld=40, codes=64, stride=128, fmt=F8, scales=64, ss=1, dw=64, lddw=100, ws=1024, size=need):
        return L.dybit_checkpoint_wgrad(T, N, K, P(dY), t, ld, P(codes), stride, fmt, P(scales), ss, P(dw), lddw, P(ws), size, None)
    assert wgrad(fmt=F4) == UNSUPPORTED
    assert wgrad(ld=39) == INVALID and wgrad(lddw=99) == INVALID and wgrad(dw=0) == INVALID and wgrad(dY=0) == INVALID and wgrad(scales=0) == INVALID
    assert wgrad(ws=0) == WORKSPACE and wgrad(size=need - 1) == WORKSPACE and wgrad(ws=1040) == ALIGNMENT and wgrad(dY=65) == ALIGNMENT


def test_plan_and_adapter_arguments():
    plan = L.dybit_adapters_plan_bytes
    assert plan(0, 1) > 0 and plan(100, 4096) > 0
    assert plan(-1, 1) == 0 and plan(10, 0) == 0 and plan(10, 4097) == 0
    assert L.dybit_adapters_plan(10, P(64), 2, P(64), plan(10, 2) - 1, None) == WORKSPACE
    assert L.dybit_adapters_plan(10, P(0), 2, P(64), plan(10, 2), None) == INVALID
    assert L.dybit_adapters_plan(10, P(64), 2, P(72), plan(10, 2), None) == ALIGNMENT

    def run(T=10, K=64, N=48, R=16, x=64, tx=BF16, ldx=64, n=2, A=64, B=64, tw=BF16, alpha=64, plan=64, base=64, ldb=48, ty=F32, y=64, ldy=48, v=64):
        return L.dybit_adapters(T, K, N, R, P(x), tx, ldx, n, P(A), P(B), tw, P(alpha), P(plan), P(base), ldb, ty, P(y), ldy, P(v), None)
    assert run(R=12) == UNSUPPORTED and run(R=136) == UNSUPPORTED and run(R=0) == INVALID and run(K=0) == INVALID
    for tx, tw, ty in ((BF16, F16, F32), (F16, BF16, F32), (F32, F16, F32), (F32, BF16, BF16), (BF16, BF16, F16), (BF16, F32, F32)):
        assert run(tx=tx, tw=tw, ty=ty) == UNSUPPORTED, (tx, tw, ty)
    assert run(ldx=63) == INVALID and run(ldy=47) == INVALID and run(ldb=47) == INVALID and run(A=0) == INVALID and run(x=0) == INVALID
    assert run(v=72) == ALIGNMENT and run(x=65) == ALIGNMENT and run(plan=72) == ALIGNMENT
    assert run(T=0) == OK


def test_backward_arguments():
    size = L.dybit_adapters_backward_workspace_bytes
    need = size(10, 64, 48, 16, 2)
    assert need > 0 and size(10, 64, 48, 12, 2) == 0 and size(10, 0, 48, 16, 2) == 0

    def run(T=10, K=64, N=48, R=16, dY=64, t=BF16, ldy=48, codes=64, stride=128, fmt=F8, scales=64, ss=1, n=2, A=64, B=64, tw=BF16, alpha=64, plan=64,
            V=64, base=64, ldb=64, dx=64, ldx=64, dA=64, dB=64, ws=1024, size=need):
        return L.dybit_adapters_backward(T, K, N, R, P(dY), t, ldy, P(codes), stride, fmt, P(scales), ss, n, P(A), P(B), tw, P(alpha), P(plan), P(V),
                                         P(base), ldb, P(dx), ldx, P(dA), P(dB), P(ws), size, None)
    assert run(t=F16) == UNSUPPORTED and run(tw=F16) == UNSUPPORTED and run(fmt=F4) == UNSUPPORTED
    assert run(dA=0) == INVALID and run(V=0) == INVALID and run(dx=0) == INVALID and run(ldx=63) == INVALID and run(stride=48) == INVALID
    assert run(ws=0) == WORKSPACE and run(size=need - 1) == WORKSPACE and run(ws=1040) == ALIGNMENT


def test_workspace_grows_with_the_problem():
    size = L.dybit_adapters_backward_workspace_bytes
    assert size(8192, 4096, 4096, 16, 4) >= size(1024, 4096, 4096, 16, 4) >= size(1024, 1024, 1024, 16, 4)
    # an adapter count beyond the tokens costs nothing but its counters
    assert size(16, 64, 64, 8, 4096) < size(16, 64, 64, 8, 16) + (1 << 20)


def test_binding_checks_its_tensors():
    cpu = torch.zeros((4, 64))
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_save(cpu, (8, 1))
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_load(torch.zeros((4, 128), dtype=torch.uint8), 64, (8, 1), torch.zeros(4))
    with pytest.raises(ValueError):
        dy.dybit_adapters_plan(torch.zeros(4, dtype=torch.int32), 2)


def test_header_documents_every_new_call():
    import os
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dybit.h")).read()
    for name in ("dybit_checkpoint_save", "dybit_checkpoint_load", "dybit_checkpoint_wgrad", "dybit_adapters_plan", "dybit_adapters",
                 "dybit_adapters_backward"):
        assert re.search(r"\b%s\(" % name, header) and hasattr(dy, name)
