"""8-bit activation checkpoints on the GPU: codes and scales bit for bit against the CPU oracle's encoder with the
row scales computed here from the definition, the activation read back, and the weight gradient against its definition
in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2302_12510_b200 as dy
from oracle import dybit_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def activation(rows, cols, seed, dtype=torch.float32, signed=True, pad=0):
    """A view [rows][cols] of a buffer with `pad` more columns; rows of very different magnitude."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols + pad), generator=g) * torch.exp(1.5 * torch.randn((rows, 1), generator=g))
    x = x * (1 + 9 * (torch.rand((1, cols + pad), generator=g) < 0.03))
    if not signed:
        x = x.relu()
    return x.to(dtype).to(DEV)[:, :cols]


def row_scales(x, top):
    """2^(ceil(log2 amax) - top) from the largest finite magnitude of each row, in exact arithmetic."""
    x = np.abs(x.astype(np.float64))
    amax = np.where(np.isfinite(x), x, 0.0).max(axis=1) if x.shape[1] else np.zeros(x.shape[0])
    mant, e = np.frexp(amax)
    e = np.clip(e - (mant == 0.5) - top, -126, 126)
    return np.where(amax > 0, np.ldexp(1.0, e), 1.0).astype(np.float32)


def check_save(x, signed, top, stride=None):
    rows, cols = x.shape
    codes_buf = None
    if stride is not None:
        codes_buf = torch.full((rows, stride), 0xAB, dtype=torch.uint8, device=DEV)
    codes, scales = dy.dybit_checkpoint_save(x, (8, signed), top=top, codes=codes_buf)
    torch.cuda.synchronize()
    xs = x.float().cpu().numpy()
    want_s = row_scales(xs, top)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    want = np.zeros((rows, codes.shape[1]), dtype=np.uint8)
    for r in range(rows):
        want[r, :cols] = orc.quantize(xs[r], 8, signed, np.float32(1.0) / want_s[r])
    got = codes.cpu().numpy()
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
    return codes, scales, want, want_s


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 4096, 0), (3, 17, 0), (5, 1000, 3), (9, 1024, 8), (4, 1025, 1), (2, 2047, 0),
                                           (3, 4097, 2), (2, 8192, 0), (2, 8200, 0), (33, 129, 7), (2, 20011, 5)])
def test_save_matches_the_oracle(dtype, rows, cols, pad):
    for signed in (True, False):
        check_save(activation(rows, cols, rows * 7 + cols, dtype, True, pad), signed, top=2 if signed else 3)


@pytest.mark.parametrize("signed,top", [(True, 0), (True, 6), (False, 0), (False, 7), (True, 4)])
def test_save_every_range_position(signed, top):
    check_save(activation(17, 300, 5), signed, top)


def test_save_every_midpoint():
    # every code value, every midpoint of neighbours, and one fp32 step to either side of both, in a row whose scale is 1
    for signed in (True, False):
        top = 6 if signed else 7
        v = np.sort(np.abs(orc.decode_table(8, signed)))
        pts = np.concatenate([v, (v[1:] + v[:-1]) / 2]).astype(np.float32)
        pts = np.concatenate([pts, np.nextafter(pts, np.float32(np.inf)), np.nextafter(pts, np.float32(0))])
        pts = np.minimum(pts, np.float32(2.0 ** top))
        x = np.stack([np.concatenate([pts, -pts, [np.float32(2.0 ** top)]])]).astype(np.float32)
        codes, scales, _, _ = check_save(torch.from_numpy(x).to(DEV), signed, top)
        assert float(scales[0]) == 1.0


def test_special_values():
    inf, nan = float("inf"), float("nan")
    rows = [[0.0] * 40, [nan] * 40, [inf, -inf, nan, 1.0, -3.0] * 8, [1e-45, -1e-45, 0.0, 1e-40] * 10,
            [3.4e38, -3.4e38, 1e38, 1.0] * 10, [-0.0, 0.0] * 20, [inf] * 40, [2.0 ** -120, 2.0 ** -126] * 20, [-1.0, -2.0] * 20]
    x = torch.tensor(rows, dtype=torch.float32, device=DEV)
    for signed in (True, False):
        for top in (0, 2, 6):
            check_save(x, signed, top)
            check_save(torch.cat([x, x.new_full((len(rows), 9000), 0.25)], dim=1), signed, top)      # the row does not fit registers
    check_save(x.to(torch.bfloat16), True, 2)
    check_save(x.to(torch.float16), True, 2)


def test_padding_is_code_zero_and_nothing_else_is_written():
    x = activation(6, 100, 3)
    big = torch.full((8, 256), 0xAB, dtype=torch.uint8, device=DEV)
    codes, scales = dy.dybit_checkpoint_save(x, (8, True), codes=big[1:7, :128])
    torch.cuda.synchronize()
    b = big.cpu().numpy()
    assert (b[1:7, 100:128] == 0).all() and (b[1:7, 128:] == 0xAB).all() and (b[0] == 0xAB).all() and (b[7] == 0xAB).all()


@pytest.mark.parametrize("out_dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (5, 1000, 3), (3, 4096, 0), (7, 777, 8), (2, 20011, 0)])
def test_load_is_scale_times_value(out_dtype, rows, cols, pad):
    g = torch.Generator().manual_seed(cols)
    codes = torch.randint(0, 256, (rows, (cols + 127) // 128 * 128), generator=g, dtype=torch.uint8)
    scales = torch.exp2(torch.randint(-8, 6, (rows,), generator=g).float())
    odd = torch.rand(rows, generator=g) + 0.1                                   # not powers of two: one fp32 product
    for signed in (True, False):
        table = torch.from_numpy(orc.decode_table(8, signed).astype(np.float32))
        for s in (scales, odd):
            buf = torch.full((rows, cols + pad), -7.0, dtype=out_dtype, device=DEV)
            y = dy.dybit_checkpoint_load(codes.to(DEV), cols, (8, signed), s.to(DEV), out=buf[:, :cols])
            want = (table[codes[:, :cols].long()] * s[:, None]).to(out_dtype)
            assert torch.equal(y.cpu(), want)
            assert (buf[:, cols:] == -7.0).all()
        pair = torch.tensor([0.37, 1 / 0.37], device=DEV)
        y = dy.dybit_checkpoint_load(codes.to(DEV), cols, (8, signed), pair, dtype=out_dtype, per_row=False)
        assert torch.equal(y.cpu(), (table[codes[:, :cols].long()] * pair[0].cpu()).to(out_dtype))


def test_load_reads_what_quantize_pack_2d_wrote():
    x = activation(9, 300, 11)
    packed, scale = dy.dybit_quantize_pack_2d(x.contiguous(), (8, 1))
    y = dy.dybit_checkpoint_load(packed, 300, (8, 1), scale, per_row=False)
    assert torch.equal(y.reshape(-1), torch.cat([dy.dybit_decode(packed[r], 300, (8, 1), scale) for r in range(9)]))


def test_empty():
    x = torch.empty((0, 64), device=DEV)
    codes, scales = dy.dybit_checkpoint_save(x, (8, True))
    assert codes.shape == (0, 128) and scales.numel() == 0
    codes, scales = dy.dybit_checkpoint_save(torch.empty((5, 0), device=DEV), (8, True), codes=torch.empty((5, 16), dtype=torch.uint8, device=DEV))
    assert (scales == 1).all()


# ---------------------------------------------------------------- weight gradient

def wgrad_case(T, N, K, dtype, signed, seed, tensor_scale=False, pad=0):
    g = torch.Generator().manual_seed(seed)
    dY = (torch.randn((T, N + pad), generator=g) * torch.exp(torch.randn((T, 1), generator=g))).to(dtype)[:, :N].to(DEV)
    x = activation(T, K, seed + 1, signed=signed)
    if tensor_scale:
        codes, pair = dy.dybit_quantize_pack_2d(x.contiguous(), (8, signed))
        return dY, codes, pair, pair[:1].expand(T)
    codes, scales = dy.dybit_checkpoint_save(x, (8, signed))
    # the padding of the rows is never part of a result
    codes[:, K:] = 0x7f
    return dY, codes, scales, scales


def check_wgrad(T, N, K, dtype, signed=True, seed=0, tensor_scale=False, pad=0, out=None):
    dY, codes, scales, s = wgrad_case(T, N, K, dtype, signed, seed, tensor_scale, pad)
    dW = dy.dybit_checkpoint_wgrad(dY, codes, K, (8, signed), scales, out=out, per_row=not tensor_scale)
    torch.cuda.synchronize()
    assert dy.dybit_last_device_status() == (0, 0)
    table = torch.from_numpy(orc.decode_table(8, signed)).to(DEV)
    X = table[codes[:, :K].long()] * s.double()[:, None]
    want = dY.double().t() @ X
    # products are exact in fp32 up to one rounding; T additions, each off by at most one fp32 step (cut off or rounded) of
    # the running sum of magnitudes
    bound = (T + 8) * 2.0 ** -23 * (dY.double().abs().t() @ X.abs()) + 1e-37
    err = (dW.double() - want).abs()
    assert (err <= bound).all(), float((err - bound).max())
    if T > 0:
        assert float(err.norm()) <= 1e-5 * float(want.norm())
    return dW


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,N,K", [(1, 1, 1), (1, 64, 64), (3, 129, 65), (17, 100, 300), (32, 1000, 512), (63, 256, 256), (64, 256, 256), (65, 257, 255),
                                   (197, 768, 768), (300, 40, 1000), (1000, 333, 77), (130, 8, 2049), (515, 520, 264)])
def test_wgrad(dtype, T, N, K):
    check_wgrad(T, N, K, dtype, signed=(T + K) % 2 == 0, seed=T + N + K)


def test_wgrad_large_sizes_in_both_dimensions():
    check_wgrad(2048, 1536, 2304, torch.bfloat16, seed=1)
    check_wgrad(700, 4100, 1028, torch.float32, seed=2)


def test_wgrad_scale_of_the_whole_tensor():
    for dtype in DTYPES:
        check_wgrad(200, 136, 264, dtype, seed=3, tensor_scale=True)


def test_wgrad_strided_gradient_and_output():
    for pad in (1, 4, 8):
        for dtype in DTYPES:
            buf = torch.full((131, 204), -7.0, device=DEV)
            check_wgrad(150, 131, 200, dtype, seed=pad, pad=pad, out=buf[:, :200])
            assert (buf[:, 200:] == -7.0).all()


def test_wgrad_of_nothing_is_zero():
    dW = dy.dybit_checkpoint_wgrad(torch.empty((0, 40), device=DEV), torch.empty((0, 128), dtype=torch.uint8, device=DEV), 70, (8, True),
                                   torch.empty(0, device=DEV), out=torch.full((40, 70), 3.0, device=DEV))
    assert (dW == 0).all()


def test_wgrad_infinities_stay_in_their_rows():
    T, N, K = 100, 70, 90
    for dtype in DTYPES:
        dY, codes, scales, s = wgrad_case(T, N, K, dtype, True, 5)
        codes[:, :K] |= 1                                              # no zero code: inf * 0 does not occur
        dY = dY.clone()
        dY[40, 3] = float("inf")
        dY[41, 5] = float("nan")
        dW = dy.dybit_checkpoint_wgrad(dY, codes, K, (8, True), scales)
        assert torch.isinf(dW[3]).all() and torch.isnan(dW[5]).all()
        rest = [i for i in range(N) if i not in (3, 5)]
        assert torch.isfinite(dW[rest]).all()


def test_wgrad_equals_differences_of_the_loss():
    # L(W) = sum(G * (X W^T)) is linear in W: its difference between two W is the gradient's product with their difference
    T, N, K = 90, 50, 70
    dY, codes, scales, _ = wgrad_case(T, N, K, torch.float32, True, 9)
    X = dy.dybit_checkpoint_load(codes, K, (8, True), scales).double()
    g = torch.Generator().manual_seed(1)
    W0, W1 = (torch.randn((N, K), generator=g, dtype=torch.float64).to(DEV) for _ in range(2))
    loss = lambda W: (dY.double() * (X @ W.t())).sum()
    dW = dy.dybit_checkpoint_wgrad(dY, codes, K, (8, True), scales).double()
    scale = (dY.double().abs().t() @ X.abs() * (W1 - W0).abs()).sum()
    assert abs(float(loss(W1) - loss(W0) - (dW * (W1 - W0)).sum())) <= float(scale) * T * 2.0 ** -22


def test_wgrad_on_another_stream_and_repeated():
    dY, codes, scales, _ = wgrad_case(400, 300, 520, torch.bfloat16, True, 21)
    a = dy.dybit_checkpoint_wgrad(dY, codes, 520, (8, True), scales)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = dy.dybit_checkpoint_wgrad(dY, codes, 520, (8, True), scales)
    s.synchronize()
    assert torch.equal(a, b)


def test_refusals():
    x = torch.zeros((4, 64), device=DEV)
    for bad in (dict(fmt=(4, 1)), dict(fmt=(8, 1), top=7), dict(fmt=(8, 0), top=8), dict(fmt=(8, 1), top=-1)):
        with pytest.raises(dy.DybitError):
            dy.dybit_checkpoint_save(x, **bad)
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_save(x.double(), (8, 1))
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_save(x.t(), (8, 1))
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_save(x, (8, 1), codes=torch.zeros((4, 48), dtype=torch.uint8, device=DEV))
    with pytest.raises(dy.DybitError):
        dy.dybit_checkpoint_save(x, (8, 1), codes=torch.zeros((4, 72), dtype=torch.uint8, device=DEV))     # row stride not a multiple of 16
    codes, scales = dy.dybit_checkpoint_save(x, (8, 1))
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_load(codes, 200, (8, 1), scales)
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_load(codes, 64, (8, 1), scales[:2].contiguous())
    with pytest.raises(dy.DybitError):
        dy.dybit_checkpoint_load(codes, 64, (6, 1), scales)
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_wgrad(x[:3], codes, 64, (8, 1), scales)
    with pytest.raises(ValueError):
        dy.dybit_checkpoint_wgrad(x, codes, 64, (8, 1), scales, out=torch.zeros((64, 60), device=DEV))
    launches = dy.dybit_launch_count()
    with pytest.raises(dy.DybitError):
        dy.dybit_checkpoint_wgrad(x, codes, 64, (8, 1), scales, ws=torch.zeros(1024, dtype=torch.uint8, device=DEV)[:8])
    assert dy.dybit_launch_count() == launches
