"""Fine-tunes and serves one linear layer whose weights are 4-bit DyBit codes.

The layer y = x W^T stays frozen as codes (dybit_gemm); a low-rank adapter beside it is trained.  What the backward pass
needs of the layer's input is kept in 8 bits (dybit_checkpoint_save).  Afterwards the tokens of several requests, each
with its own adapter or none, go through the layer in one call.  A second run trains the weights themselves, with the
gradient read from the same kind of checkpoint (dybit_checkpoint_wgrad) and fake quantization in front of the product.

    python examples/finetune_coded_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2302_12510_b200 as dy  # noqa: E402

W_FMT, X_FMT = (4, True), (8, True)


def coded_product(x, codes_w, scale_w, N):
    """x W^T on coded operands: the activation takes 8-bit codes with one scale for the tensor."""
    T, K = x.shape
    codes_x, scale_x = dy.dybit_quantize_pack_2d(x, X_FMT)
    y, _ = dy.dybit_gemm(T, N, K, codes_x, X_FMT, scale_x, codes_w, W_FMT, scale_w)
    return y


def train_adapter(T=512, K=256, N=192, R=16, steps=60, lr=1.0, seed=0, device="cuda"):
    """Returns (losses, A, B): a rank-R adapter that learns what separates the coded layer from a target layer."""
    g = torch.Generator(device=device).manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device=device)
    W = randn(N, K) / K ** 0.5
    codes_w, scale_w = dy.dybit_quantize_pack_2d(W, W_FMT)
    target_delta = randn(N, R) @ randn(R, K) / (K * R) ** 0.5
    A, B = randn(1, R, K) / K ** 0.5, torch.zeros((1, R, N), device=device)      # fp32 masters, bf16 copies in the calls
    plan = dy.AdapterPlan(torch.zeros(T, dtype=torch.int32, device=device), 1)
    losses = []
    for _ in range(steps):
        x = randn(T, K)
        target = x @ (W + target_delta).t()
        a, b = A.bfloat16(), B.bfloat16()
        base = coded_product(x, codes_w, scale_w, N)
        y, v = dy.dybit_adapters(x, a, b, None, plan, base, out=base, want_v=True)
        codes, scales = dy.dybit_checkpoint_save(x, X_FMT, top=2)                # all that is kept of x
        error = y - target
        losses.append(float((error * error).mean()))
        dY = error * (2.0 / T)
        _, dA, dB = dy.dybit_adapters_backward(dY, codes, X_FMT, scales, a, b, None, plan, v)
        A -= lr * dA / N
        B -= lr * dB
    return losses, A, B


def train_weights(T=512, K=256, N=192, steps=40, lr=0.5, seed=0, device="cuda"):
    """Quantization-aware training of the weights: fake-quantized forward, straight-through gradient."""
    g = torch.Generator(device=device).manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device=device)
    goal, W = randn(N, K) / K ** 0.5, torch.zeros((N, K), device=device)
    W += 0.1 * randn(N, K) / K ** 0.5
    losses = []
    for _ in range(steps):
        x = randn(T, K)
        scale_w = dy.dybit_absmax_scale(W, (8, True))
        codes, scales = dy.dybit_checkpoint_save(x, X_FMT, top=2)
        error = x @ dy.dybit_fake_quant(W, (8, True), scale_w).t() - x @ goal.t()
        losses.append(float((error * error).mean()))
        dW = dy.dybit_checkpoint_wgrad(error * (1.0 / T), codes, K, X_FMT, scales)
        W -= lr * dy.dybit_fake_quant_backward(W, dW, (8, True), scale_w)
    return losses


def serve(A, B, T=24, seed=1, device="cuda"):
    """One decode step of T requests: half of them with the trained adapter, some with an untrained one, some with none."""
    R, K, N = A.shape[1], A.shape[2], B.shape[2]
    g = torch.Generator(device=device).manual_seed(seed)
    x = torch.randn((T, K), generator=g, device=device)
    codes_w, scale_w = dy.dybit_quantize_pack_2d(torch.randn((N, K), generator=g, device=device) / K ** 0.5, W_FMT)
    ids = torch.tensor([(0, 1, 0, -1)[t % 4] for t in range(T)], dtype=torch.int32, device=device)
    a = torch.cat([A, torch.randn((1, R, K), generator=g, device=device) / K ** 0.5]).bfloat16()
    b = torch.cat([B, torch.zeros((1, R, N), device=device)]).bfloat16()
    plan = dy.AdapterPlan(ids, 2)                            # one plan for every projection of every layer of this step
    base = coded_product(x, codes_w, scale_w, N)
    y, _ = dy.dybit_adapters(x, a, b, None, plan, base)
    return base, y, ids


def main():
    losses, A, B = train_adapter()
    print("adapter: loss %.4f -> %.4f" % (losses[0], losses[-1]))
    base, y, ids = serve(A, B)
    print("served %d tokens, %d of them changed by their adapter" % (len(ids), int((y != base).any(dim=1).sum())))
    losses = train_weights()
    print("weights: loss %.4f -> %.4f" % (losses[0], losses[-1]))


if __name__ == "__main__":
    main()
