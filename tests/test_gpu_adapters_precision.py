"""The adapters' second product in full fp32: V enters it with all its bits and the base is added to the finished sum,
whatever the types of y and of the factors.

The cases make V exact and the rest cancel, so that nothing hides an error of the product.  V = a0 + x1 * a1 has 24
significant bits and is a sum of two products that fp32 holds exactly; one rank is not zero; the base is -V * b rounded to
its type.  Bound: V as an operand 2^-24, two additions of the tensor core's parts 2^-23 each (it may cut off), both of
|V * b|, and y's own rounding, half a step of y.  (Two truncated bf16 parts would be off by up to 2^-15 of |V * b|, two
truncated tf32 parts by up to 2^-21.)"""
import pytest
import torch

import paper_2302_12510_b200 as dy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, H, F = torch.bfloat16, torch.float16, torch.float32
EPS = {F: 2.0 ** -24, BF: 2.0 ** -8, H: 2.0 ** -11}          # half a step at most: 24, 8 and 11 significant bits


def cancelling(T, K, N, R, tx, ty, seed):
    """x, A, B, base and the exact V * b of rank 3, for one adapter."""
    g = torch.Generator().manual_seed(seed)
    u = lambda n, steps: (1 + torch.randint(0, steps, (n,), generator=g) / steps).double()     # [1, 2) in `steps` steps
    tw = H if tx == H else BF
    x, A, B = torch.zeros(T, K).double(), torch.zeros(1, R, K).double(), torch.zeros(1, R, N).double()
    x[:, 1] = 1.0
    if tx == H:                                              # steps of 2^-10 in V's upper half, of 2^-22 in all
        A[0, 3, 1], A[0, 3, K - 1] = u(1, 1024)[0], 1.75
        x[:, K - 1] = u(T, 1024) * 2.0 ** -10
        B[0, 3] = u(N, 1024)
    else:                                                    # steps of 2^-7, and of 2^-22 in all
        A[0, 3, 1], A[0, 3, K - 1] = u(1, 128)[0], u(1, 128)[0]
        x[:, K - 1] = u(T, 128) * 2.0 ** -8
        B[0, 3] = u(N, 128)
    v = x @ A[0, 3]
    vb = v[:, None] * B[0, 3][None, :]
    base = (-vb).to(ty)
    for t, w, d in ((x, tx, "x"), (A, tw, "A"), (B, tw, "B")):
        assert torch.equal(t.to(w).double(), t), d
    assert torch.equal(v.float().double(), v)
    return x.to(tx).to(DEV), A.to(tw).to(DEV), B.to(tw).to(DEV), base.to(DEV), vb.to(DEV)


def check(y, base, vb):
    want = base.double() + vb
    bound = (2.0 ** -24 + 2 * 2.0 ** -23) * vb.abs() + EPS[y.dtype] * (want.abs() + 2.0 ** -21 * vb.abs()) + 2.0 ** -25
    err = (y.double() - want).abs()
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("tx,ty", [(BF, BF), (BF, F), (H, H), (H, F), (F, F)])
@pytest.mark.parametrize("T,K,N,R", [(1, 64, 64, 8), (7, 100, 135, 16), (70, 256, 200, 16), (33, 128, 264, 32), (20, 72, 64, 64), (17, 64, 128, 128)])
def test_forward_where_base_and_adapter_cancel(tx, ty, T, K, N, R):
    x, A, B, base, vb = cancelling(T, K, N, R, tx, ty, seed=T + N + R)
    plan = dy.AdapterPlan(torch.zeros(T, dtype=torch.int32, device=DEV), 1)
    y, _ = dy.dybit_adapters(x, A, B, None, plan, base)
    check(y, base, vb)


@pytest.mark.parametrize("t", [BF, F])
@pytest.mark.parametrize("T,K,N,R", [(1, 64, 64, 8), (40, 136, 100, 16), (70, 200, 256, 32)])
def test_backward_where_base_and_adapter_cancel(t, T, K, N, R):
    # dX = dXbase + U A is the same operator with the factors exchanged
    dY, B, A, base, vb = cancelling(T, N, K, R, t, t, seed=T + N + R)
    plan = dy.AdapterPlan(torch.zeros(T, dtype=torch.int32, device=DEV), 1)
    codes, scales = dy.dybit_checkpoint_save(torch.ones((T, K), device=DEV), (8, True))
    dx, _, _ = dy.dybit_adapters_backward(dY, codes, (8, True), scales, A, B, None, plan, torch.zeros((T, R), device=DEV), base)
    check(dx, base, vb)


@pytest.mark.parametrize("ty", [BF, H, F])
def test_token_without_adapter_keeps_its_base_bit_for_bit(ty):
    tx = H if ty == H else BF
    base = torch.tensor([0.0, -0.0, 1.5, -2.25, float("inf"), float("-inf"), 2.0 ** -14, -2.0 ** -20] * 8, device=DEV).to(ty).repeat(3, 1)
    x, A, B = torch.ones((3, 64), device=DEV).to(tx), torch.ones((1, 8, 64), device=DEV).to(tx), torch.ones((1, 8, 64), device=DEV).to(tx)
    plan = dy.AdapterPlan(torch.tensor([-1, -1, 7], dtype=torch.int32, device=DEV), 1)
    y, _ = dy.dybit_adapters(x, A, B, None, plan, base)
    bits = torch.int32 if ty == F else torch.int16
    assert torch.equal(y.view(bits), base.view(bits))


def test_gradient_products_of_fp32_numbers():
    # one token, so dB is one product of two fp32 numbers, each in three bf16 parts.  Numbers 1 + n * 2^-23 for every n below
    # 2^16: their leading part is 1, the rest is all in the lower parts.  Bound, relative to the product (which is at least 1):
    # two products of lower parts that are left out, 2^-23 each, and additions that may cut off, 2^-23 in the last and less than
    # a 64th of it in the others
    N, R = 1 << 16, 8
    dY = (1 + torch.arange(N, device=DEV).double() * 2.0 ** -23).float()[None]
    v = (1 + torch.tensor([0xffff, 0x8000, 0xff80, 0x7f80, 0x0080, 0x7fff, 0xff7f, 0x5555], device=DEV).double() * 2.0 ** -23).float()[None]
    plan = dy.AdapterPlan(torch.zeros(1, dtype=torch.int32, device=DEV), 1)
    codes, scales = dy.dybit_checkpoint_save(torch.ones((1, 64), device=DEV), (8, True))
    A, B = torch.zeros((1, R, 64), dtype=BF, device=DEV), torch.zeros((1, R, N), dtype=BF, device=DEV)
    _, _, dB = dy.dybit_adapters_backward(dY, codes, (8, True), scales, A, B, None, plan, v)
    want = v[0].double()[:, None] * dY[0].double()[None, :]
    err = ((dB[0].double() - want) / want).abs()
    assert float(err.max()) <= (2 + 1 + 2.0 ** -6) * 2.0 ** -23, float(err.max()) * 2.0 ** 23
