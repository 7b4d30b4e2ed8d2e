"""Infinities and NaN in the adapters' backward pass: each gradient has them exactly where its definition in 64 bits has
them, with the same signs, and everything else keeps its bits."""
import pytest
import torch

import paper_2302_12510_b200 as dy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def case(T, K, N, R, t, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)
    n = 3
    s = dict(A=(r(n, R, K) / K ** 0.5).to(BF).to(DEV), B=r(n, R, N).to(BF).to(DEV), alpha=(0.5 + torch.rand(n, generator=g)).to(DEV),
             dY=(0.1 * r(T, N)).to(t).to(DEV), v=r(T, R).to(DEV), dxb=r(T, K).to(t).to(DEV))
    s["ids"] = (torch.arange(T) % 4 - 1).to(torch.int32).to(DEV)        # adapters 0, 1, 2 and none in turn
    s["plan"] = dy.AdapterPlan(s["ids"], n)
    s["codes"], s["scales"] = dy.dybit_checkpoint_save(r(T, K).to(DEV), (8, True))
    s["X"] = dy.dybit_checkpoint_load(s["codes"], K, (8, True), s["scales"])
    return s


def run(s):
    out = dy.dybit_adapters_backward(s["dY"], s["codes"], (8, True), s["scales"], s["A"], s["B"], s["alpha"], s["plan"], s["v"], s["dxb"])
    torch.cuda.synchronize()
    assert dy.dybit_last_device_status() == (0, 0)
    return out


def want(s):
    """(dX, dA, dB) by the formulas, summed in 64 bits one token after the other (a matrix product may skip or pad)."""
    dY, A, B, alpha, v, X = (s[k].double() for k in ("dY", "A", "B", "alpha", "v", "X"))
    dx, dA, dB = s["dxb"].double().clone(), torch.zeros_like(A), torch.zeros_like(B)
    for t, a in enumerate(s["ids"].tolist()):
        if a < 0:
            continue
        U = alpha[a] * (B[a] * dY[t][None, :]).sum(dim=1)
        dx[t] += (U[:, None] * A[a]).sum(dim=0)
        dA[a] += U[:, None] * X[t][None, :]
        dB[a] += alpha[a] * v[t][:, None] * dY[t][None, :]
    return dx, dA, dB


def same_kind(got, w, clean):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(w))
    assert torch.equal(torch.isinf(got), torch.isinf(w))
    assert torch.equal(got[torch.isinf(w)], w[torch.isinf(w)])
    fine = torch.isfinite(w)
    assert torch.equal(got[fine], clean.double()[fine])


@pytest.mark.parametrize("t", [BF, F])
@pytest.mark.parametrize("T,K,N,R", [(21, 64, 64, 8), (130, 200, 136, 16), (130, 77, 131, 16), (70, 128, 320, 32), (70, 130, 67, 32),
                                     (45, 72, 128, 64), (600, 64, 70, 16), (45, 64, 77, 128)])
def test_infinities_and_nan_in_the_gradient(t, T, K, N, R):
    s = case(T, K, N, R, t, seed=T + K + N + R)
    # short products of the forward pass that have few significant bits: their lower parts are zeros
    s["v"][5], s["v"][9], s["v"][10] = 1.0, -0.375, 0.0
    s["dY"][9, 7] = 0.5
    clean = run(s)
    dY = s["dY"]
    dY[5, 3] = INF                                             # adapter 0
    dY[9, 4], dY[9, 6] = -INF, INF                             # adapter 0
    dY[13, 6] = INF                                            # adapter 0: two infinities of one column
    dY[10, 8] = INF                                            # adapter 1, with a V of zero: 0 * infinity
    dY[14, 9] = NAN                                            # adapter 1
    dY[4, 10], dY[8, 11] = INF, NAN                            # no adapter
    got = run(s)
    for g, w, c in zip(got, want(s), clean):
        same_kind(g, w, c)
    assert torch.isfinite(got[1][2]).all() and torch.isfinite(got[2][2]).all()         # adapter 2 had none


@pytest.mark.parametrize("t", [BF, F])
@pytest.mark.parametrize("T,K,N,R", [(21, 64, 64, 8), (130, 77, 131, 16), (70, 128, 320, 32), (45, 72, 128, 64)])
def test_infinities_in_the_short_product(t, T, K, N, R):
    # V of a forward pass that ran over, against gradients with few significant bits
    s = case(T, K, N, R, t, seed=T + K)
    s["dY"][6, :8] = torch.tensor([0.5, -0.5, 1.0, 0.0, 2.0, -4.0, 0.25, 3.0])
    clean = run(s)
    s["v"][6, 1], s["v"][6, 2], s["v"][7, 0] = INF, -INF, NAN
    got = run(s)
    for g, w, c in zip(got, want(s), clean):
        same_kind(g, w, c)
