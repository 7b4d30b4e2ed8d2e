"""Measured cases of the language-model operators: 8-bit activation checkpoints and low-rank adapters.

A linear layer whose weights are DyBit codes is trained and served with four operators beside its coded product:

  checkpoint         an activation is stored as 8-bit DyBit codes with one power-of-two scale per row, and read back
  wgrad              the weight gradient dW = dY^T X^ of a linear layer, X^ read from those codes
  adapters           y = base + alpha_a * (x A_a^T) B_a for the tokens of many requests, each with its own adapter a
  adapters_backward  dX, dA and dB of the same, x read from an 8-bit checkpoint

`own` chooses between the plain form (elementary torch operations in 32 bits) and the library's calls.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_DEV = "cuda:0"


# ---------------------------------------------------------------- cases

def listed():
    return [
        # the input of the classifier of a ResNet-18 at batch 32: 512 features after a ReLU, hence unsigned codes
        dict(name="checkpoint 32x512 f32 unsigned", kind="checkpoint", rows=32, cols=512, pad=0, dtype="f32", signed=False, top=2),
        # a ragged slice of a wider buffer: odd sizes, rows that start on odd 4-byte boundaries
        dict(name="checkpoint 1999x1003 f32 strided", kind="checkpoint", rows=1999, cols=1003, pad=4, dtype="f32", signed=True, top=3),
        # the input of one projection of a 4096-wide layer for 16384 tokens of a training batch
        dict(name="checkpoint 16384x4096 bf16", kind="checkpoint", rows=16384, cols=4096, pad=0, dtype="bf16", signed=True, top=2),
        # the classifier of a ResNet-18 at batch 32: few rows, launch latency counts
        dict(name="wgrad 32x1000x512 bf16", kind="wgrad", T=32, N=1000, K=512, dtype="bf16", signed=False),
        # a square projection of a ViT-Base, batch 8 of 197 tokens, gradients kept in 32 bits
        dict(name="wgrad 1576x768x768 f32", kind="wgrad", T=1576, N=768, K=768, dtype="f32", signed=True),
        # a square projection of a 4096-wide layer, 8192 tokens: one large matrix product
        dict(name="wgrad 8192x4096x4096 bf16", kind="wgrad", T=8192, N=4096, K=4096, dtype="bf16", signed=True),
        # one token of one request: latency of a single decode step
        dict(name="adapters 1 token", kind="adapters", T=1, K=4096, N=4096, R=16, n=1, dtype="bf16", ydtype="bf16", order="mixed", none=0.0, save_v=False),
        # a decode step of 256 requests over 64 adapters beside an fp32 product, an eighth of them without an adapter
        dict(name="adapters 256 tokens of 64", kind="adapters", T=256, K=4096, N=4096, R=16, n=64, dtype="bf16", ydtype="f32", order="mixed", none=0.125, save_v=False),
        # odd sizes throughout, half precision
        dict(name="adapters ragged f16", kind="adapters", T=1001, K=1003, N=777, R=8, n=5, dtype="f16", ydtype="f16", order="runs", none=0.1, save_v=False),
        # the forward pass of a training step (or a prefill): 8192 tokens of 8 requests in 32 bits, the short product kept
        dict(name="adapters 8192 tokens f32", kind="adapters", T=8192, K=4096, N=4096, R=16, n=8, dtype="f32", ydtype="f32", order="runs", none=0.0, save_v=True),
        # the backward pass of a small layer: one image of a ViT-Base, one adapter
        dict(name="backward 197 tokens f32", kind="adapters_backward", T=197, K=768, N=768, R=8, n=1, dtype="f32", order="runs", none=0.0, signed=True),
        # the backward pass of the training step above in 16 bits, four adapters trained side by side
        dict(name="backward 8192 tokens bf16", kind="adapters_backward", T=8192, K=4096, N=4096, R=16, n=4, dtype="bf16", order="runs", none=0.0, signed=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A feature count: half of them multiples of 64, as layers have them, the rest anything."""
    v = _log_int(rng, lo, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["checkpoint", "wgrad", "adapters", "adapters_backward"])
    most = max((work(c) for c in listed() if c["kind"] == kind), key=lambda w: w["bytes"] + w["flops"] / 50)
    while True:
        if kind == "checkpoint":
            c = dict(kind=kind, rows=_log_int(rng, 1, 16384), cols=_width(rng, 64, 8192), pad=rng.choice([0, 0, 1, 8]),
                     dtype=rng.choice(["f32", "bf16", "f16"]), signed=rng.random() < 0.7, top=rng.randint(1, 4))
        elif kind == "wgrad":
            c = dict(kind=kind, T=_log_int(rng, 1, 8192), N=_width(rng, 64, 4096), K=_width(rng, 64, 4096),
                     dtype=rng.choice(["f32", "bf16", "f16"]), signed=rng.random() < 0.7)
        else:
            t, width = _log_int(rng, 1, 8192), (_width(rng, 64, 4096), _width(rng, 64, 4096))
            c = dict(kind=kind, T=t, K=width[0], N=width[1], R=rng.choice([8, 16, 24, 32, 64]), n=_log_int(rng, 1, 64))
            if kind == "adapters":
                c["dtype"] = rng.choice(["f32", "bf16", "f16"])
                c["ydtype"] = rng.choice(["f32", c["dtype"]])
                c["save_v"] = rng.random() < 0.5
            else:
                c["dtype"] = rng.choice(["f32", "bf16"])
                c["signed"] = rng.random() < 0.7
            c["order"] = rng.choice(["mixed", "runs"])
            c["none"] = rng.choice([0.0, 0.1])
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


def _padded(cols):
    return (cols + 127) // 128 * 128


def work(case):
    """Bytes read and written once, and the multiplications and additions of the products."""
    if case["kind"] == "checkpoint":
        n = case["rows"] * case["cols"]
        # the activation is read, its codes written; later the codes are read and the activation written
        return {"bytes": n * (2 * _BYTES[case["dtype"]] + 2) + 8 * case["rows"], "flops": 4 * n}
    T, N, K = case["T"], case["N"], case["K"]
    e = _BYTES[case["dtype"]]
    if case["kind"] == "wgrad":
        return {"bytes": T * N * e + T * K + 4 * T + 4 * N * K, "flops": 2 * T * N * K}
    R, used = case["R"], min(case["n"], T)
    if case["kind"] == "adapters":
        y = _BYTES[case["ydtype"]]
        return {"bytes": T * K * e + 2 * T * N * y + used * R * (K + N) * 2 + 4 * T + (4 * T * R if case["save_v"] else 0),
                "flops": 2 * T * R * (K + N)}
    return {"bytes": T * N * e + T * K + 2 * T * K * e + 8 * T + 4 * T * R + used * R * (K + N) * 2 + case["n"] * R * (K + N) * 4,
            "flops": 4 * T * R * (K + N)}


# ---------------------------------------------------------------- the 8-bit format in plain form

def _pow2(e):
    """2^e for an int32 tensor of exponents -126..126."""
    return ((e + 127) << 23).view(torch.float32)


def _row_scales(x, top):
    """The power of two that takes a row's largest finite magnitude into (2^(top-1), 2^top]; 1 for a row of zeros."""
    a = x.float().abs()
    amax = torch.where(torch.isfinite(a), a, torch.zeros_like(a)).amax(dim=1)
    mant, e = torch.frexp(amax)
    e = e.to(torch.int32) - (mant == 0.5).to(torch.int32)
    s = _pow2((e - top).clamp(-126, 126))
    return torch.where(amax > 0, s, torch.ones_like(s))


def _encode(x, scales, signed):
    """8-bit codes of x / scale: nearest value, ties to the even code, NaN to code 0."""
    m = 7 if signed else 8
    x = x.float() * (1.0 / scales)[:, None]
    t = x.abs() if signed else x
    t = torch.where(t > 0, t, torch.zeros_like(t)).clamp(max=2.0 ** (m - 1))
    low = torch.round(t * 2.0 ** (m - 1)).to(torch.int32)
    e = (torch.frexp(t.clamp(min=1.0))[1] - 1).to(torch.int32).clamp(0, m - 2)
    k = m - 2 - e
    high = (1 << m) - (2 << k) + torch.round(t * _pow2(k - e) - (1 << k)).to(torch.int32)
    mag = torch.where(t < 1, low, high).clamp(max=(1 << m) - 1)
    code = mag + 128 * ((x < 0) & (mag > 0)).to(torch.int32) if signed else mag
    return code.to(torch.uint8)


def _values(signed, dtype, device):
    """The value of each of the 256 codes: leading ones are the exponent, the bits below the first zero the fraction."""
    m = 7 if signed else 8
    c = torch.arange(1 << m, device=device)
    ones = sum(((c >> (m - 1 - i)) == (2 << i) - 1).long() for i in range(m))
    k = (m - 1 - ones).clamp(min=0)
    frac = (c & ((1 << k) - 1)).to(dtype) / (1 << k).to(dtype)
    v = torch.where(ones > 0, (2.0 ** (ones - 1).to(dtype)) * (1 + frac), c.to(dtype) / 2 ** (m - 1))
    v = torch.where(ones == m, torch.full_like(v, 2.0 ** (m - 1)), v)
    return torch.cat([v, -v]) if signed else v


def _decode(codes, scales, values):
    return values[codes.long()] * scales[:, None]


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device=_DEV).manual_seed(int(seed))


def _activation(g, rows, cols, signed):
    """Rows of different magnitude with a few strong channels, as activations have them; non-negative after a ReLU."""
    x = torch.randn((rows, cols), generator=g, device=_DEV)
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=g, device=_DEV))
    x *= 1 + 7 * (torch.rand((1, cols), generator=g, device=_DEV) < 0.01)
    return x if signed else x.relu_()


def _checkpoint(g, rows, cols, signed):
    """Codes and scales of a stored activation, rows padded with code 0 to a multiple of 128 codes."""
    x = _activation(g, rows, cols, signed)
    scales = _row_scales(x, 2)
    codes = torch.zeros((rows, _padded(cols)), dtype=torch.uint8, device=_DEV)
    codes[:, :cols] = _encode(x, scales, signed)
    return codes, scales


def _ids(g, T, n, order, none):
    """The adapter of each token (-1: none): every token on its own, or runs of tokens of one request."""
    if order == "mixed":
        ids = torch.randint(0, n, (T,), generator=g, device=_DEV)
        ids = torch.where(torch.rand((T,), generator=g, device=_DEV) < none, torch.full_like(ids, -1), ids)
        return ids.to(torch.int32)
    runs = max(1, min(T, 2 * n))
    cuts = torch.randint(0, T, (runs - 1,), generator=g, device=_DEV).sort()[0]
    run = torch.searchsorted(cuts, torch.arange(T, device=_DEV), right=True)
    of = torch.randperm(runs, generator=g, device=_DEV) % n
    of = torch.where(torch.rand((runs,), generator=g, device=_DEV) < none, torch.full_like(of, -1), of)
    return of[run].to(torch.int32)


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case=case)
    if own:
        import paper_2302_12510_b200 as dy
        s["dy"] = dy
    elif case.get("signed") is not None:
        s["values"] = _values(case["signed"], torch.float32, _DEV)
    dt = _DTYPES[case["dtype"]]
    if case["kind"] == "checkpoint":
        wide = _activation(g, case["rows"], case["cols"] + case["pad"], case["signed"]).to(dt)
        s["x"] = wide[:, :case["cols"]]
        return s
    T, N, K = case["T"], case["N"], case["K"]
    if case["kind"] == "wgrad":
        s["dy_"] = (1e-2 * torch.randn((T, N), generator=g, device=_DEV)).to(dt)
        s["codes"], s["scales"] = _checkpoint(g, T, K, case["signed"])
        return s
    n, R = case["n"], case["R"]
    wt = torch.float16 if case["dtype"] == "f16" else torch.bfloat16
    s["A"] = (torch.randn((n, R, K), generator=g, device=_DEV) / math.sqrt(K)).to(wt)
    s["B"] = (0.1 * torch.randn((n, R, N), generator=g, device=_DEV)).to(wt)
    s["alpha"] = 0.5 + torch.rand((n,), generator=g, device=_DEV)
    s["ids"] = _ids(g, T, n, case["order"], case["none"])
    if own:
        # built once per batch of tokens: every projection of every layer goes by the same plan
        s["plan"] = s["dy"].AdapterPlan(s["ids"], n)
    if case["kind"] == "adapters":
        s["x"] = _activation(g, T, K, True).to(dt)
        s["base"] = torch.randn((T, N), generator=g, device=_DEV).to(_DTYPES[case["ydtype"]])
    else:
        s["dy_"] = (1e-2 * torch.randn((T, N), generator=g, device=_DEV)).to(dt)
        s["dx_base"] = (1e-2 * torch.randn((T, K), generator=g, device=_DEV)).to(dt)
        s["codes"], s["scales"] = _checkpoint(g, T, K, case["signed"])
        s["v"] = torch.randn((T, R), generator=g, device=_DEV)
        s["v"][s["ids"] < 0] = 0
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    c, dy = s["case"], s["dy"]
    if c["kind"] == "checkpoint":
        fmt = (8, c["signed"])
        codes, scales = dy.dybit_checkpoint_save(s["x"], fmt, top=c["top"])
        return {"y": dy.dybit_checkpoint_load(codes, c["cols"], fmt, scales, dtype=s["x"].dtype), "scales": scales}
    if c["kind"] == "wgrad":
        return dy.dybit_checkpoint_wgrad(s["dy_"], s["codes"], c["K"], (8, c["signed"]), s["scales"])
    if c["kind"] == "adapters":
        y, v = dy.dybit_adapters(s["x"], s["A"], s["B"], s["alpha"], s["plan"], s["base"], want_v=c["save_v"])
        return {"y": y, "v": v} if c["save_v"] else y
    dx, dA, dB = dy.dybit_adapters_backward(s["dy_"], s["codes"], (8, c["signed"]), s["scales"], s["A"], s["B"], s["alpha"],
                                            s["plan"], s["v"], s["dx_base"])
    return {"dx": dx, "dA": dA, "dB": dB}


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "checkpoint":
        scales = _row_scales(s["x"], c["top"])
        return {"y": _decode(_encode(s["x"], scales, c["signed"]), scales, s["values"]).to(s["x"].dtype), "scales": scales}
    if c["kind"] == "wgrad":
        x = _decode(s["codes"][:, :c["K"]], s["scales"], s["values"])
        return s["dy_"].float().t() @ x
    # all adapters at once, each token keeping the columns of its own
    T, n, R = c["T"], c["n"], c["R"]
    A, B = s["A"].float().view(n * R, c["K"]), s["B"].float().view(n * R, c["N"])
    mine = (s["ids"][:, None] == torch.arange(n, device=_DEV)[None, :])[:, :, None]
    nothing = torch.zeros((), device=_DEV)

    def keep(v):
        return torch.where(mine, v.view(T, n, R), nothing)

    scaled = torch.where(mine, s["alpha"][None, :, None], nothing)
    if c["kind"] == "adapters":
        v = keep(s["x"].float() @ A.t())
        y = (s["base"].float() + (v * scaled).view(T, n * R) @ B).to(s["base"].dtype)
        return {"y": y, "v": v.sum(dim=1)} if c["save_v"] else y
    dY = s["dy_"].float()
    x = _decode(s["codes"][:, :c["K"]], s["scales"], s["values"])
    u = (keep(dY @ B.t()) * scaled).view(T, n * R)
    v = (s["v"][:, None, :] * scaled).view(T, n * R)
    return {"dx": (s["dx_base"].float() + u @ A).to(s["dx_base"].dtype), "dA": (u.t() @ x).view(n, R, c["K"]),
            "dB": (v.t() @ dY).view(n, R, c["N"])}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_values(signed):
    """Value of each code from the format's definition, one code after the other."""
    m, out = (7 if signed else 8), []
    for code in range(256):
        c = code & ((1 << m) - 1)
        bits = format(c, "0%db" % m)
        run_ = len(bits) - len(bits.lstrip("1"))
        rest = bits[run_ + 1:]
        if run_ == 0:
            v = c / 2 ** (m - 1)
        elif run_ == m:
            v = 2.0 ** (m - 1)
        else:
            v = 2.0 ** (run_ - 1) * (1 + (int(rest, 2) / 2 ** len(rest) if rest else 0.0))
        out.append(-v if signed and code >> m else v)
    return torch.tensor(out, dtype=torch.float64, device=_DEV)


def _exact_checkpoint(s):
    c, x = s["case"], s["x"].double()
    values = _exact_values(c["signed"])
    table = values[:128] if c["signed"] else values
    amax = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(dim=1)
    scale = torch.where(amax > 0, torch.exp2(torch.round(torch.ceil(torch.log2(amax) - 1e-12)).clamp(min=-200) - c["top"]),
                        torch.ones_like(amax))
    t = x / scale[:, None]
    mag = (t.abs() if c["signed"] else t.clamp(min=0)).clamp(max=float(table[-1])).contiguous()
    hi = torch.searchsorted(table, mag).clamp(1, len(table) - 1)
    below, above = mag - table[hi - 1], table[hi] - mag
    pick = torch.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, hi - 1)
    y = table[pick] * scale[:, None]
    return {"y": torch.where(x < 0, -y, y) if c["signed"] else y, "scales": scale}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "checkpoint":
        return _exact_checkpoint(s)
    x = None if case["kind"] == "adapters" else _exact_values(case["signed"])[s["codes"][:, :case["K"]].long()] * s["scales"].double()[:, None]
    if case["kind"] == "wgrad":
        return torch.einsum("tn,tk->nk", s["dy_"].double(), x)
    n, R = case["n"], case["R"]
    A, B, alpha = s["A"].double(), s["B"].double(), s["alpha"].double()
    of = [torch.nonzero(s["ids"] == a)[:, 0] for a in range(n)]
    if case["kind"] == "adapters":
        y, v = s["base"].double(), torch.zeros((case["T"], R), dtype=torch.float64, device=_DEV)
        for a, at in enumerate(of):
            v[at] = s["x"][at].double() @ A[a].t()
            y[at] += alpha[a] * (v[at] @ B[a])
        return {"y": y, "v": v} if case["save_v"] else y
    dY, dx, dA, dB = s["dy_"].double(), s["dx_base"].double(), torch.zeros_like(A), torch.zeros_like(B)
    for a, at in enumerate(of):
        u = alpha[a] * (dY[at] @ B[a].t())
        dx[at] += u @ A[a]
        dA[a] = u.t() @ x[at]
        dB[a] = alpha[a] * (s["v"][at].double().t() @ dY[at])
    return {"dx": dx, "dA": dA, "dB": dB}
