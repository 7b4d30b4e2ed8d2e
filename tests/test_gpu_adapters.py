"""Low-rank adapters of many requests on the GPU: forward and gradients against the definition in 64 bits.

Tolerances.  V is a sum of K products in fp32, each addition off by at most one fp32 step of the running sum of
magnitudes; y adds R products of V (cut into two tf32 numbers: relative error 2^-21) and the base, and is rounded once
to its type.  The gradients are sums over the tokens of products with U, which is a sum like V."""
import pytest
import torch

import paper_2302_12510_b200 as dy
from oracle import dybit_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a step: 24, 8 and 11 significant bits
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}
BF, H, F = torch.bfloat16, torch.float16, torch.float32


def make(T, K, N, R, n, tx, ty, seed, ids=None, pad=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)
    tw = H if tx == H else BF
    s = dict(x=r(T, K + pad).to(tx).to(DEV)[:, :K], A=(r(n, R, K) / K ** 0.5).to(tw).to(DEV), B=r(n, R, N).to(tw).to(DEV),
             alpha=(0.5 + torch.rand(n, generator=g)).to(DEV), base=r(T, N + pad).to(ty).to(DEV)[:, :N])
    if ids is None:
        ids = torch.randint(-1, n, (T,), generator=g)
    s["ids"] = torch.as_tensor(ids, dtype=torch.int32).to(DEV)
    s["plan"] = dy.AdapterPlan(s["ids"], n)
    return s


def forward_want(s):
    """(y, V, bound of y, bound of V) in 64 bits; rows of x that are not finite make NaN here and there: see the tests."""
    x, A, B, alpha = s["x"].double(), s["A"].double(), s["B"].double(), s["alpha"].double()
    base = s["base"].double()
    y, ty = base.clone(), s["base"].dtype
    V = torch.zeros((x.shape[0], A.shape[1]), dtype=torch.float64, device=DEV)
    bv, by = torch.zeros_like(V), torch.zeros_like(y)
    K, R = A.shape[2], A.shape[1]
    for a in range(A.shape[0]):
        at = torch.nonzero(s["ids"] == a)[:, 0]
        V[at] = x[at] @ A[a].t()
        bv[at] = (K + 8) * 2.0 ** -23 * (x[at].abs() @ A[a].abs().t())
        y[at] += alpha[a] * (V[at] @ B[a])
        by[at] = alpha[a] * ((bv[at] + (R + 8) * 2.0 ** -21 * V[at].abs()) @ B[a].abs())
    by = by + 2.0 ** -23 * base.abs() + EPS[ty] * (y.abs() + by) + TINY[ty]
    return y, V, by, bv + 1e-37


def check_forward(s, in_place=False, want_v=True):
    y, V, by, bv = forward_want(s)
    base = s["base"]
    out = None
    if in_place:
        out = base = base.clone()
    got, v = dy.dybit_adapters(s["x"], s["A"], s["B"], s["alpha"], s["plan"], base, out=out, want_v=want_v)
    torch.cuda.synchronize()
    assert dy.dybit_last_device_status() == (0, 0)
    assert got.dtype == s["base"].dtype
    assert ((got.double() - y).abs() <= by).all(), float(((got.double() - y).abs() - by).max())
    if want_v:
        assert ((v.double() - V).abs() <= bv).all()
    none = (s["ids"] < 0) | (s["ids"] >= s["A"].shape[0])
    assert torch.equal(got[none], s["base"][none])
    return got, v


TYPES = [(BF, BF), (BF, F), (H, H), (H, F), (F, F)]


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("T,K,N,R,n", [(1, 64, 64, 16, 1), (1, 1, 1, 8, 1), (2, 4096, 100, 16, 3), (5, 65, 63, 8, 2), (16, 512, 512, 32, 1),
                                       (17, 1003, 777, 8, 5), (40, 300, 1000, 24, 3), (64, 128, 260, 64, 64), (33, 72, 520, 128, 2),
                                       (256, 1024, 640, 16, 40)])
def test_forward_tokens_of_many_requests(tx, ty, T, K, N, R, n):
    check_forward(make(T, K, N, R, n, tx, ty, seed=T + K + N + R + n))


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("R", [8, 16, 24, 32, 48, 64, 96, 128])
def test_forward_long_runs_every_rank(tx, ty, R):
    T, n = 333, 3
    ids = torch.cat([torch.full((150,), 2), torch.full((3,), -1), torch.full((180,), 0)])       # adapter 1 has no token
    check_forward(make(T, 456, 392, R, n, tx, ty, seed=R, ids=ids))


def test_forward_strided_rows_and_in_place():
    for tx, ty in TYPES:
        for pad in (1, 2, 8):
            check_forward(make(70, 200, 136, 16, 2, tx, ty, seed=pad, pad=pad))
        check_forward(make(70, 200, 136, 16, 2, tx, ty, seed=3), in_place=True)


def test_forward_without_base_alpha_or_tokens():
    s = make(20, 128, 96, 16, 2, BF, F, seed=1)
    got, v = dy.dybit_adapters(s["x"], s["A"], s["B"], None, s["plan"], out_dtype=F)
    assert v is None
    s2 = dict(s, base=torch.zeros_like(s["base"]), alpha=torch.ones_like(s["alpha"]))
    y, _, by, _ = forward_want(s2)
    assert ((got.double() - y).abs() <= by).all()
    e = make(0, 128, 96, 16, 2, BF, F, seed=1)
    got, v = dy.dybit_adapters(e["x"], e["A"], e["B"], e["alpha"], e["plan"], e["base"], want_v=True)
    assert got.shape == (0, 96) and v.shape == (0, 16)


def test_forward_all_tokens_without_adapter_and_foreign_ids():
    s = make(100, 128, 96, 16, 2, BF, BF, seed=1, ids=torch.full((100,), -1))
    got, v = check_forward(s)
    assert (v == 0).all()
    ids = torch.randint(-5, 9, (100,), generator=torch.Generator().manual_seed(0))
    ids[3] = 2 ** 31 - 1
    ids[4] = -2 ** 31
    s = make(100, 128, 96, 16, 2, BF, BF, seed=1, ids=ids)
    check_forward(s)


def test_forward_rows_that_are_not_finite_stay_alone():
    for tx, ty in TYPES:
        s = make(90, 200, 136, 16, 2, tx, ty, seed=4)
        clean, _ = dy.dybit_adapters(s["x"], s["A"], s["B"], s["alpha"], s["plan"], s["base"])
        s["x"][7] = float("nan")
        s["x"][8, 5] = float("inf")
        s["ids"][7] = s["ids"][8] = 1
        s["ids"][9] = -1
        s["x"][9] = float("inf")
        s["base"][10, 0] = float("-inf")
        s["plan"] = dy.AdapterPlan(s["ids"], 2)
        got, v = dy.dybit_adapters(s["x"], s["A"], s["B"], s["alpha"], s["plan"], s["base"], want_v=True)
        assert torch.isnan(got[7]).all() and torch.equal(got[9], s["base"][9]) and (v[9] == 0).all()
        # one infinity: V is an infinity of the factor's sign, as the sum in fp32 gives it
        assert torch.equal(v[8], float("inf") * s["A"][1, :, 5].float().sign())
        assert got[10, 0] == float("-inf")
        rest = [i for i in range(90) if i not in (7, 8, 9, 10)]
        assert torch.equal(got[rest], clean[rest])


def test_forward_same_bits_for_any_order_of_requests():
    # a token's result does not depend on where in the batch it stands
    s = make(64, 512, 256, 16, 8, BF, F, seed=6)
    a, _ = dy.dybit_adapters(s["x"], s["A"], s["B"], s["alpha"], s["plan"], s["base"])
    p = torch.randperm(64, generator=torch.Generator().manual_seed(2)).to(DEV)
    plan = dy.AdapterPlan(s["ids"][p].contiguous(), 8)
    b, _ = dy.dybit_adapters(s["x"][p].contiguous(), s["A"], s["B"], s["alpha"], plan, s["base"][p].contiguous())
    assert torch.equal(a[p], b)


# ---------------------------------------------------------------- gradients

def make_backward(T, K, N, R, n, t, seed, ids=None, pad=0, signed=True, tensor_scale=False):
    s = make(T, K, N, R, n, F if t == F else BF, F, seed, ids)
    g = torch.Generator().manual_seed(seed + 1000)
    r = lambda *sh: torch.randn(sh, generator=g)
    x = r(T, K) * torch.exp(r(T, 1))
    x = (x if signed else x.relu()).to(DEV)
    if tensor_scale:
        s["codes"], s["scales"] = dy.dybit_quantize_pack_2d(x, (8, signed))
        s["row"] = s["scales"][:1].expand(T)
    else:
        s["codes"], s["scales"] = dy.dybit_checkpoint_save(x, (8, signed))
        s["row"] = s["scales"]
        s["codes"][:, K:] = 0x55
    s["fmt"], s["per_row"] = (8, signed), not tensor_scale
    s["dY"] = (0.1 * r(T, N + pad)).to(t).to(DEV)[:, :N]
    s["dxb"] = (0.1 * r(T, K + pad)).to(t).to(DEV)[:, :K]
    s["v"] = r(T, R).to(DEV)
    return s


def backward(s, **kw):
    return dy.dybit_adapters_backward(s["dY"], s["codes"], s["fmt"], s["scales"], s["A"], s["B"], s["alpha"], s["plan"], s["v"], s["dxb"],
                                      per_row=s["per_row"], **kw)


def check_backward(s):
    dx, dA, dB = backward(s)
    torch.cuda.synchronize()
    assert dy.dybit_last_device_status() == (0, 0)
    T, N = s["dY"].shape
    K, R = s["A"].shape[2], s["A"].shape[1]
    table = torch.from_numpy(orc.decode_table(8, bool(s["fmt"][1]))).to(DEV)
    X = table[s["codes"][:, :K].long()] * s["row"].double()[:, None]
    dY, A, B, alpha = s["dY"].double(), s["A"].double(), s["B"].double(), s["alpha"].double()
    wx, bx = s["dxb"].double().clone(), torch.zeros_like(s["dxb"].double())
    for a in range(A.shape[0]):
        at = torch.nonzero(s["ids"] == a)[:, 0]
        U = alpha[a] * (dY[at] @ B[a].t())
        bu = alpha[a] * (N + 10) * 2.0 ** -23 * (dY[at].abs() @ B[a].abs().t())
        wx[at] += U @ A[a]
        bx[at] = (bu + (R + 8) * 2.0 ** -21 * U.abs()) @ A[a].abs()
        m = at.numel()
        wa, wb = U.t() @ X[at], alpha[a] * (s["v"][at].double().t() @ dY[at])
        ba = bu.t() @ X[at].abs() + (m + 12) * 2.0 ** -22 * (U.abs().t() @ X[at].abs()) + 1e-37
        bb = alpha[a] * (m + 12) * 2.0 ** -22 * (s["v"][at].double().abs().t() @ dY[at].abs()) + 1e-37
        assert ((dA[a].double() - wa).abs() <= ba).all(), ("dA", a)
        assert ((dB[a].double() - wb).abs() <= bb).all(), ("dB", a)
        if m == 0:
            assert (dA[a] == 0).all() and (dB[a] == 0).all()
        else:
            assert float((dA[a].double() - wa).norm()) <= 1e-5 * float(wa.norm())
            assert float((dB[a].double() - wb).norm()) <= 1e-5 * float(wb.norm())
    t = s["dY"].dtype
    bx = bx + 2.0 ** -23 * s["dxb"].double().abs() + EPS[t] * (wx.abs() + bx) + TINY[t]
    assert ((dx.double() - wx).abs() <= bx).all()
    return dx, dA, dB


@pytest.mark.parametrize("t", [BF, F])
@pytest.mark.parametrize("T,K,N,R,n", [(1, 64, 64, 16, 1), (1, 1, 1, 8, 1), (3, 130, 66, 8, 2), (17, 1003, 777, 8, 5), (50, 200, 300, 24, 4),
                                       (64, 128, 260, 64, 64), (130, 72, 520, 128, 2), (197, 768, 768, 8, 1), (200, 264, 136, 32, 3),
                                       (257, 256, 512, 48, 2)])
def test_backward(t, T, K, N, R, n):
    check_backward(make_backward(T, K, N, R, n, t, seed=T + K + N + R + n, signed=(T % 2 == 0)))


@pytest.mark.parametrize("t", [BF, F])
def test_backward_adapters_of_many_tokens(t):
    # adapters with one chunk of tokens, several, and none
    ids = torch.cat([torch.full((1300,), 2), torch.full((5,), -1), torch.full((512,), 0), torch.full((513,), 3), torch.full((7,), 2)])
    check_backward(make_backward(ids.numel(), 200, 328, 16, 5, t, seed=8, ids=ids[torch.randperm(ids.numel(), generator=torch.Generator().manual_seed(3))]))


def test_backward_strides_and_scale_of_the_whole_tensor():
    for t in (BF, F):
        for pad in (1, 4, 8):
            check_backward(make_backward(70, 200, 136, 16, 2, t, seed=pad, pad=pad))
        check_backward(make_backward(70, 200, 136, 16, 2, t, seed=3, tensor_scale=True))
        check_backward(make_backward(70, 203, 135, 16, 2, t, seed=3, tensor_scale=True, signed=False))


def test_backward_of_nothing():
    for T, ids in ((0, []), (40, [-1] * 40)):
        s = make_backward(T, 128, 96, 16, 2, BF, seed=1, ids=torch.tensor(ids, dtype=torch.int32))
        dA, dB = (torch.full(s[k].shape, 3.0, device=DEV) for k in "AB")
        dx, dA, dB = backward(s, dA=dA, dB=dB)
        assert torch.equal(dx, s["dxb"]) and (dA == 0).all() and (dB == 0).all()


def test_backward_in_place_repeated_and_on_another_stream():
    s = make_backward(700, 264, 136, 16, 3, BF, seed=5)
    a = backward(s)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b = backward(s, dx=s["dxb"].clone())
        c = s["dxb"].clone()
        s2 = dict(s, dxb=c)
        b2 = backward(s2, dx=c)
    st.synchronize()
    for u, w, z in zip(a, b, b2):
        assert torch.equal(u, w) and torch.equal(u, z)


def test_backward_equals_differences_of_the_forward_pass():
    # y is linear in A, in B and in x: the loss sum(G * y) differs between two factors by the gradient's product with their
    # difference.  The forward pass runs on the activation that the checkpoint stands for.
    T, K, N, R, n = 60, 128, 96, 16, 2
    s = make_backward(T, K, N, R, n, F, seed=12)
    x = dy.dybit_checkpoint_load(s["codes"], K, s["fmt"], s["scales"])
    G = s["dY"]
    zero = torch.zeros((T, N), device=DEV)

    def forward(x, A, B):
        return dy.dybit_adapters(x, A, B, s["alpha"], s["plan"], zero, want_v=True)

    def loss(x, A, B):
        return float((G.double() * forward(x, A, B)[0].double()).sum())

    _, s["v"] = forward(x, s["A"], s["B"])
    s["dxb"] = torch.zeros_like(s["dxb"])
    dx, dA, dB = backward(s)
    g = torch.Generator().manual_seed(77)
    A1, B1 = ((s[k].float() + 0.3 * torch.randn(s[k].shape, generator=g).to(DEV)).to(BF) for k in "AB")
    x1 = x + torch.randn(x.shape, generator=g).to(DEV)
    for got, want, size in ((loss(x, A1, s["B"]) - loss(x, s["A"], s["B"]), dA.double() * (A1.double() - s["A"].double()), dA.abs().double()),
                            (loss(x, s["A"], B1) - loss(x, s["A"], s["B"]), dB.double() * (B1.double() - s["B"].double()), dB),
                            (loss(x1, s["A"], s["B"]) - loss(x, s["A"], s["B"]), dx.double() * (x1.double() - x.double()), dx)):
        magnitude = (G.double().abs() * forward(x.abs(), s["A"].abs(), s["B"].abs())[0].double()).sum() + want.abs().sum()
        assert abs(got - float(want.sum())) <= 2.0 ** -20 * float(magnitude)


def test_plan_groups_tokens_in_order():
    # through the operators' own eyes: rank-8 adapters that copy one column, so V tells which factor a token met
    T, n = 3000, 700
    ids = torch.randint(-1, n, (T,), generator=torch.Generator().manual_seed(9))
    x = torch.ones((T, 8), device=DEV)
    A = torch.zeros((n, 8, 8), dtype=BF, device=DEV)
    A[:, 0, 0] = torch.arange(n, device=DEV).to(BF)                    # bf16 rounds, the same way below
    B = torch.zeros((n, 8, 8), dtype=BF, device=DEV)
    plan = dy.AdapterPlan(ids.to(torch.int32).to(DEV), n)
    _, v = dy.dybit_adapters(x, A, B, None, plan, torch.zeros((T, 8), device=DEV), want_v=True)
    want = torch.where(ids >= 0, torch.arange(n).to(BF).float()[ids.clamp(min=0)], torch.zeros(()))
    assert torch.equal(v[:, 0].cpu(), want)


def test_refusals():
    s = make(20, 128, 96, 16, 2, BF, F, seed=1)
    go = lambda **kw: dy.dybit_adapters(*[{**s, **kw}[k] for k in ("x", "A", "B", "alpha", "plan", "base")])
    launches = dy.dybit_launch_count()
    with pytest.raises(dy.DybitError):
        go(x=s["x"].to(H))                                             # 16-bit types that differ
    with pytest.raises(dy.DybitError):
        go(base=s["base"].to(H))
    with pytest.raises(dy.DybitError):
        go(A=s["A"][:, :12].contiguous(), B=s["B"][:, :12].contiguous())     # rank not a multiple of 8
    with pytest.raises(dy.DybitError):
        go(A=torch.zeros((2, 136, 128), dtype=BF, device=DEV), B=torch.zeros((2, 136, 96), dtype=BF, device=DEV))
    for bad in (dict(x=s["x"][:, :100]), dict(x=s["x"][:10]), dict(B=s["B"][:1].contiguous()), dict(A=s["A"].float(), B=s["B"].float()),
                dict(alpha=s["alpha"][:1].contiguous()), dict(base=s["base"][:, :90]), dict(x=s["x"].t())):
        with pytest.raises(ValueError):
            go(**bad)
    assert dy.dybit_launch_count() == launches
    with pytest.raises(dy.DybitError):
        dy.dybit_adapters_plan(s["ids"], 0, plan=torch.zeros(4096, dtype=torch.uint8, device=DEV))
    with pytest.raises(dy.DybitError):
        dy.dybit_adapters_plan(s["ids"], 5000, plan=torch.zeros(4096, dtype=torch.uint8, device=DEV))
    with pytest.raises(dy.DybitError):
        dy.dybit_adapters_plan(s["ids"], 2, plan=torch.zeros(64, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        dy.dybit_adapters_plan(s["ids"].long(), 2)
    b = make_backward(20, 128, 96, 16, 2, BF, seed=1)
    with pytest.raises(dy.DybitError):
        backward(dict(b, dY=b["dY"].to(H), dxb=b["dxb"].to(H)))
    with pytest.raises(dy.DybitError):
        backward(b, ws=torch.zeros(2048, dtype=torch.uint8, device=DEV)[:1100])
    with pytest.raises(ValueError):
        backward(dict(b, v=b["v"][:, :8]))
