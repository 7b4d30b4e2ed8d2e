"""Refusals of the fine-tuning operators that come before the first launch, however large the problem."""
import ctypes

import pytest
import torch

import paper_2302_12510_b200 as dy

L = dy.lib
P = ctypes.c_void_p
F8 = dy.binding._CFmt(8, 1)
UNSUPPORTED, WORKSPACE = 2, 4
BF16 = 1


@pytest.mark.parametrize("T,n", [(40_000_000, 2), (65535 * 512, 1), ((65535 - 2 * 4096 + 1) * 512, 4096)])
def test_backward_of_more_tokens_than_its_grid_holds(T, n):
    # dX (which may be dXbase itself) is written by the first of two kernels: the second one's limit is looked at before it.
    # The addresses are stand-ins; nothing is launched
    K, N, R = 64, 48, 16
    need = L.dybit_adapters_backward_workspace_bytes(T, K, N, R, n)
    launches = dy.dybit_launch_count()
    st = L.dybit_adapters_backward(T, K, N, R, P(64), BF16, N, P(64), 128, F8, P(64), 1, n, P(64), P(64), BF16, P(64), P(64), P(64), P(64), K, P(64), K,
                                   P(64), P(64), P(1024), need, None)
    assert st == UNSUPPORTED
    assert dy.dybit_launch_count() == launches


def test_types_that_the_operators_do_not_have():
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_wgrad_workspace_bytes(32, 64, 64, torch.float64)


@pytest.mark.gpu
def test_output_types_that_the_operators_do_not_have():
    x, f = torch.zeros((4, 64), device="cuda"), torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    plan = dy.AdapterPlan(torch.zeros(4, dtype=torch.int32, device="cuda"), 2)
    with pytest.raises(ValueError):
        dy.dybit_adapters(x, f, f, None, plan, out_dtype=torch.float64)
    codes, scales = dy.dybit_checkpoint_save(x, (8, 1))
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_load(codes, 64, (8, 1), scales, dtype=torch.float64)
