"""How exact the weight gradient from a checkpoint is: over long sums, and with row scales that are no powers of two."""
import numpy as np
import pytest
import torch

import paper_2302_12510_b200 as dy
from oracle import dybit_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def decoded(codes, K, signed, scales):
    table = torch.from_numpy(orc.decode_table(8, signed).astype(np.float64)).to(DEV)
    return table[codes[:, :K].long()] * scales.double()[:, None]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,N,K", [(8192, 256, 512), (16384, 72, 130)])
def test_long_sums_are_as_exact_as_in_plain_fp32(dtype, T, N, K):
    # Limit of the relative error (2-norm).  A product in plain fp32 has 3.3e-7 for 8192 tokens as torch computes it.  An
    # accumulator that stays on the tensor core over the whole length is cut off T / 16 times and has 3.4e-6.  1e-6 lies a
    # factor of three from either.
    g = torch.Generator().manual_seed(T + N)
    dY = (0.01 * torch.randn((T, N), generator=g)).to(dtype).to(DEV)
    codes, scales = dy.dybit_checkpoint_save(torch.randn((T, K), generator=g).to(DEV), (8, True))
    dW = dy.dybit_checkpoint_wgrad(dY, codes, K, (8, True), scales)
    want = dY.double().t() @ decoded(codes, K, True, scales)
    assert float((dW.double() - want).norm()) <= 1e-6 * float(want.norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,N,K", [(1, 64, 64), (197, 130, 264), (1000, 77, 203)])
def test_row_scales_that_are_no_powers_of_two(dtype, T, N, K):
    # x^ enters the product as the bf16 number nearest to scale * value (rounded to fp32 first): off by at most 2^-8 + 2^-24 of it.
    # Beside that the sum's own error, at most one fp32 step per addition
    g = torch.Generator().manual_seed(T)
    dY = torch.randn((T, N), generator=g).to(dtype).to(DEV)
    for signed in (True, False):
        x = torch.randn((T, K), generator=g)
        codes, scales = dy.dybit_checkpoint_save((x if signed else x.abs()).to(DEV), (8, signed))
        scales = scales * (1 + torch.rand(T, generator=g).to(DEV))
        dW = dy.dybit_checkpoint_wgrad(dY, codes, K, (8, signed), scales)
        X = decoded(codes, K, signed, scales)
        want, size = dY.double().t() @ X, dY.double().abs().t() @ X.abs()
        bound = (2.0 ** -8 + 2.0 ** -24 + (T + 8) * 2.0 ** -23) * size + 1e-37
        assert ((dW.double() - want).abs() <= bound).all()
        # exactly the sum over the rounded activation
        rounded = (decoded(codes, K, signed, torch.ones_like(scales)).float() * scales[:, None]).bfloat16().double()
        want = dY.double().t() @ rounded
        assert ((dW.double() - want).abs() <= (T + 8) * 2.0 ** -23 * (dY.double().abs().t() @ rounded.abs()) + 1e-37).all()
