"""Measured cases of the key-value cache in 8-bit codes and of the attention that reads it.

A model that is served keeps the keys and values of its past tokens as signed 8-bit DyBit codes.  The cache is a pool of
pages; a page holds `page` consecutive tokens of one sequence, and each page has one power-of-two scale per head for its
keys and one for its values.  Three operators:

  write      the keys and values of new tokens are stored behind what their sequences hold already; a page that is only
             begun keeps its scale, or takes a larger one and its older codes with it
  read       tokens are read back from the cache as dense keys and values
  attention  softmax(q k^T * scale + mask) v for the new tokens of a batch of sequences, keys and values read from the cache

`own` chooses between the plain form (elementary torch operations in 32 bits) and the library's calls.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_DEV = "cuda:0"
_TOP = 2                     # a page's largest magnitude lies in (2, 4] of the code's value axis


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one token of each of 64 requests is stored: the write of a decode step, latency counts
        dict(name="write 64 requests 1 token", kind="write", B=64, chunks=0, new=1, ctx=2000, spread=True, heads=8, dim=128, page=64, dtype="bf16"),
        # four prompts of 2048 tokens behind a begun page
        dict(name="write 4 prompts of 2048", kind="write", B=4, chunks=4, new=2048, ctx=100, spread=True, heads=8, dim=128, page=64, dtype="bf16"),
        # odd sizes throughout, 32 bits, keys and values as slices of one projection's output
        dict(name="write ragged f32", kind="write", B=5, chunks=3, new=333, ctx=1000, spread=True, heads=3, dim=80, page=16, dtype="f32"),
        # the 197 tokens of one image of a ViT-Base, 12 heads of 64
        dict(name="read 197 tokens f32", kind="read", B=1, chunks=1, new=197, ctx=0, spread=False, heads=12, dim=64, page=16, dtype="f32"),
        # eight long sequences are handed on in 16 bits
        dict(name="read 8 sequences of 8192", kind="read", B=8, chunks=8, new=8192, ctx=0, spread=False, heads=8, dim=128, page=64, dtype="bf16"),
        # one token of one request: latency of a single decode step, few rows and a long axis
        dict(name="decode 1 request of 4096", kind="attention", B=1, chunks=0, new=1, ctx=4095, spread=False, heads=8, group=4, dim=128, page=64, dtype="bf16", window=0, causal=True),
        # a decode step of 64 requests with up to 8192 tokens: one pass over the cache
        dict(name="decode 64 requests to 8192", kind="attention", B=64, chunks=0, new=1, ctx=8191, spread=True, heads=8, group=4, dim=128, page=64, dtype="bf16", window=0, causal=True),
        # many short requests, a head of queries for each head of keys, small pages, half precision
        dict(name="decode 200 requests f16", kind="attention", B=200, chunks=0, new=1, ctx=2000, spread=True, heads=12, group=1, dim=64, page=16, dtype="f16", window=0, causal=True),
        # five drafted tokens of each of seven requests are checked in one pass, groups of seven heads
        dict(name="decode 7 requests 5 drafts", kind="attention", B=7, chunks=7, new=5, ctx=3001, spread=True, heads=4, group=7, dim=96, page=32, dtype="bf16", window=0, causal=True),
        # the prompt of one request, all of it at once
        dict(name="prompt of 8192", kind="attention", B=1, chunks=1, new=8192, ctx=0, spread=False, heads=8, group=4, dim=128, page=64, dtype="bf16", window=0, causal=True),
        # a chunk of each of two prompts behind a long past
        dict(name="chunks of 1000 behind 16384", kind="attention", B=2, chunks=2, new=1000, ctx=16384, spread=False, heads=4, group=8, dim=128, page=128, dtype="f16", window=0, causal=True),
        # chunks and single tokens in one batch, each token sees the last 1024
        dict(name="mixed batch, window 1024", kind="attention", B=32, chunks=2, new=500, ctx=6000, spread=True, heads=8, group=4, dim=128, page=64, dtype="bf16", window=1024, causal=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "attention", "attention"])
    most = max((work(c) for c in listed() if c["kind"] == kind), key=lambda w: w["bytes"] + w["flops"] / 50)
    while True:
        c = dict(kind=kind, B=_log_int(rng, 1, 256), heads=rng.choice([1, 2, 3, 4, 8, 12]), dim=rng.choice([64, 80, 96, 128]),
                 page=rng.choice([16, 32, 64, 128]), spread=rng.random() < 0.7)
        if kind == "read":
            c.update(chunks=c["B"], new=_log_int(rng, 1, 8192), ctx=rng.choice([0, _log_int(rng, 1, 1000)]), dtype=rng.choice(["f32", "bf16", "f16"]))
        elif kind == "write":
            c.update(chunks=rng.choice([0, rng.randint(1, c["B"]), c["B"]]), new=_log_int(rng, 1, 4096), ctx=_log_int(rng, 1, 4000),
                     dtype=rng.choice(["f32", "bf16", "f16"]))
        else:
            c.update(chunks=rng.choice([0, 0, rng.randint(1, c["B"]), c["B"]]), new=rng.choice([rng.randint(2, 8), _log_int(rng, 2, 4096)]),
                     ctx=_log_int(rng, 1, 32768), group=rng.choice([1, 2, 3, 4, 7, 8]), dtype=rng.choice(["bf16", "f16"]),
                     window=rng.choice([0, 0, _log_int(rng, 16, 4096)]), causal=rng.random() < 0.85)
            if not c["causal"]:
                c["window"] = 0
        w = work(c)
        news, lens = _lengths(c)
        rows = c["B"] * max(news) * c["heads"] * c.get("group", 1)
        held = c["B"] * max(lens) * c["heads"] * c["dim"]
        # the plain form pads: its scores and its keys have to fit the card
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and held <= 1 << 30 and (kind != "attention" or rows * max(lens) <= 1 << 31):
            return c


def _lengths(c):
    """(new tokens, tokens in all) of each sequence: the first `chunks` sequences have `new` new tokens, the others one."""
    news = [c["new"] if b < c["chunks"] else 1 for b in range(c["B"])]
    past = [int(c["ctx"] * (0.25 + 0.75 * math.modf((b + 1) * 0.6180339887)[0])) if c["spread"] else c["ctx"] for b in range(c["B"])]
    return news, [n + p for n, p in zip(news, past)]


def _touched(c):
    """Tokens of the pages that new tokens go to, from each page's first token on."""
    news, lens = _lengths(c)
    return [ln - (ln - n) // c["page"] * c["page"] for n, ln in zip(news, lens)]


def work(case):
    """Bytes read and written once, and the multiplications and additions."""
    news, lens = _lengths(case)
    e, width, T = _BYTES[case["dtype"]], case["heads"] * case["dim"], sum(news)
    if case["kind"] == "write":
        # new tokens are read and their codes written; the pages they went to are read back
        return {"bytes": T * width * 2 * (e + 1) + sum(_touched(case)) * width * 2 * (1 + e), "flops": 8 * T * width}
    if case["kind"] == "read":
        return {"bytes": T * width * 2 * (1 + e), "flops": 2 * T * width}
    seen = pairs = 0
    for n, ln in zip(news, lens):
        w = case["window"] or ln
        seen += min(ln, w + n - 1)
        first = ln - n + 1 if case["causal"] else ln
        # token i of n sees min(first + i, w) keys (all of them without a causal mask)
        full = max(0, min(n, w - first)) if case["causal"] else n
        pairs += full * first + (full * (full - 1) // 2 if case["causal"] else 0) + (n - full) * min(w, ln)
    scales = seen // case["page"] * case["heads"] * 8
    return {"bytes": T * width * case["group"] * 2 * e + seen * width * 2 + scales, "flops": 4 * pairs * width * case["group"]}


# ---------------------------------------------------------------- the 8-bit format in plain form

def _pow2(e):
    """2^e for an int32 tensor of exponents -126..126."""
    return ((e + 127) << 23).view(torch.float32)


def _scale(amax):
    """The power of two that takes amax into (2^(top-1), 2^top]; 0 for a block of zeros."""
    mant, e = torch.frexp(amax)
    e = e.to(torch.int32) - (mant == 0.5).to(torch.int32)
    s = _pow2((e - _TOP).clamp(-126, 126))
    return torch.where(amax > 0, s, torch.zeros_like(s))


def _encode(x, scale):
    """Signed 8-bit codes of x / scale: nearest value, ties to the even code, code 0 where the scale is 0."""
    x = x * torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    t = x.abs().clamp(max=64.0)
    low = torch.round(t * 64.0).to(torch.int32)
    e = (torch.frexp(t.clamp(min=1.0))[1] - 1).to(torch.int32).clamp(0, 5)
    k = 5 - e
    high = 128 - (2 << k) + torch.round(t * _pow2(k - e) - (1 << k)).to(torch.int32)
    mag = torch.where(t < 1, low, high).clamp(max=127)
    return (mag + 128 * ((x < 0) & (mag > 0)).to(torch.int32)).to(torch.uint8)


def _values(dtype=torch.float32):
    """The value of each of the 256 codes: leading ones are the exponent, the bits below the first zero the fraction."""
    c = torch.arange(128, device=_DEV)
    ones = sum(((c >> (6 - i)) == (2 << i) - 1).long() for i in range(7))
    k = (6 - ones).clamp(min=0)
    frac = (c & ((1 << k) - 1)).to(dtype) / (1 << k).to(dtype)
    v = torch.where(ones > 0, (2.0 ** (ones - 1).to(dtype)) * (1 + frac), c.to(dtype) / 64)
    v = torch.where(ones == 7, torch.full_like(v, 64.0), v)
    return torch.cat([v, -v])


# ---------------------------------------------------------------- inputs

def _keys(g, shape):
    """Keys or values: a few strong channels, tokens of different magnitude."""
    x = torch.randn(shape, generator=g, device=_DEV)
    x *= torch.exp(0.3 * torch.randn(shape[:-1] + (1,), generator=g, device=_DEV))
    return x * (1 + 4 * (torch.rand(shape[-1:], generator=g, device=_DEV) < 0.03))


def _pool(g, pages, c):
    """Codes [pages][heads][page][dim] and scales [pages][heads] of a cache in use."""
    codes = torch.empty((pages, c["heads"], c["page"], c["dim"]), dtype=torch.uint8, device=_DEV)
    scales = torch.empty((pages, c["heads"]), device=_DEV)
    step = max(1, (1 << 25) // (c["heads"] * c["page"] * c["dim"]))
    for p in range(0, pages, step):
        x = _keys(g, tuple(codes[p:p + step].shape))
        scales[p:p + step] = _scale(x.abs().amax(dim=(2, 3)))
        codes[p:p + step] = _encode(x, scales[p:p + step, :, None, None])
    return codes, scales


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=_DEV)


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    g = torch.Generator(device=_DEV).manual_seed(int(seed))
    news, lens = _lengths(case)
    B, H, D, page, T = case["B"], case["heads"], case["dim"], case["page"], sum(news)
    s = dict(case=case, T=T, values=_values())
    used = [-(-ln // page) for ln in lens]
    pages, most = sum(used) + 3, max(used)
    s["k_codes"], s["k_scales"] = _pool(g, pages, case)
    s["v_codes"], s["v_scales"] = _pool(g, pages, case)
    # the pages of a sequence lie anywhere in the pool; entries behind its last page are not looked at
    order = torch.randperm(pages, generator=g, device=_DEV).to(torch.int32)
    col = torch.arange(most, device=_DEV)[None, :]
    at, count = _ints(_starts(used))[:-1], _ints(used)
    s["table"] = torch.where(col < count[:, None], order[(at[:, None] + col).clamp(max=pages - 1)], -1).to(torch.int32).contiguous()
    s["lens"], s["starts"] = _ints(lens), _ints(_starts(news))
    dt = _DTYPES[case["dtype"]]
    group = case.get("group", 1)
    packed = _keys(g, (T, (group + 2) * H, D)).to(dt)          # what the projection of queries, keys and values gives
    s["q"], s["k"], s["v"] = packed[:, :group * H], packed[:, group * H:(group + 1) * H], packed[:, (group + 1) * H:]
    # where each token goes: kept by a program for all layers of a step
    token = torch.arange(T, device=_DEV)
    s["seq"] = torch.searchsorted(s["starts"][1:].long(), token, right=True)
    s["nth"] = token - s["starts"].long()[s["seq"]]
    s["pos"] = (s["lens"] - (s["starts"][1:] - s["starts"][:-1])).long()[s["seq"]] + s["nth"]
    if case["kind"] == "write":
        back = _touched(case)
        first = [ln - n for n, ln in zip(back, lens)]
        s["back_starts"], TR = _ints(_starts(back)), sum(back)
        token = torch.arange(TR, device=_DEV)
        seq = torch.searchsorted(s["back_starts"][1:].long(), token, right=True)
        pos = token - s["back_starts"].long()[seq] + _ints(first).long()[seq]
        s["back_page"], s["back_off"] = s["table"].long()[seq, pos // page], pos % page
        # the pages that new tokens go to, and how many tokens each holds before
        blocks = [-(-n // page) for n in back]
        base = _ints(_starts(blocks)).long()
        s["block"] = base[s["seq"]] + s["pos"] // page - _ints(first).long()[s["seq"]] // page
        block = torch.arange(sum(blocks), device=_DEV)
        owner = torch.searchsorted(base[1:], block, right=True)
        nth = block - base[owner]
        s["block_page"] = s["table"].long()[owner, _ints(first).long()[owner] // page + nth]
        before = (s["lens"] - (s["starts"][1:] - s["starts"][:-1])).long() % page
        s["before"] = torch.where(nth == 0, before[owner], torch.zeros_like(nth))
    if own:
        import paper_2302_12510_b200 as dy
        s["dy"] = dy
        s["cache"] = dy.KVCache(pages, page, H, D, k_codes=s["k_codes"], v_codes=s["v_codes"], k_scales=s["k_scales"], v_scales=s["v_scales"])
        # made once for a step: every layer's calls go by the same plan
        s["plan"] = dy.CachePlan(s["cache"], s["table"], s["starts"], s["lens"], T, q_heads=group * H, max_new=max(news))
        if case["kind"] == "write":
            s["back_plan"] = dy.CachePlan(s["cache"], s["table"], s["back_starts"], s["lens"], TR, max_new=max(back))
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    c, dy = s["case"], s["dy"]
    if c["kind"] == "write":
        dy.dybit_cache_write(s["cache"], s["k"], s["v"], s["plan"], top=_TOP)
        k, v = dy.dybit_cache_read(s["cache"], s["back_plan"], dtype=s["k"].dtype)
        return {"k": k, "v": v, "k_scales": s["k_scales"], "v_scales": s["v_scales"]}
    if c["kind"] == "read":
        k, v = dy.dybit_cache_read(s["cache"], s["plan"], dtype=s["k"].dtype)
        return {"k": k, "v": v}
    return dy.dybit_cache_attention(s["q"], s["cache"], s["plan"], causal=c["causal"], window=c["window"])


def _write_plain(s, x, codes, scales):
    c, block, off = s["case"], s["block"], s["pos"] % s["case"]["page"]
    fresh = torch.zeros((len(s["block_page"]), c["heads"], c["page"], c["dim"]), device=_DEV)
    fresh[block, :, off] = x.float()
    kept, before = codes[s["block_page"]], s["before"][:, None]
    old = torch.where(before > 0, scales[s["block_page"]], torch.zeros((), device=_DEV))
    scale = torch.maximum(old, _scale(fresh.abs().amax(dim=(2, 3))))
    ratio = (old / scale)[:, :, None, None]
    # an older code is rounded again where the scale has grown
    moved = torch.where(ratio < 1, _encode(s["values"][kept.int()] * ratio, torch.ones_like(ratio)), kept)
    row = torch.arange(c["page"], device=_DEV)[None, :]
    is_new = torch.zeros((len(s["block_page"]), c["page"]), dtype=torch.bool, device=_DEV)
    is_new[block, off] = True
    out = torch.where((row < before)[:, None, :, None], moved, kept)
    out = torch.where(is_new[:, None, :, None], _encode(fresh, scale[:, :, None, None]), out)
    codes[s["block_page"]] = out
    scales[s["block_page"]] = scale
    return (s["values"][codes[s["back_page"], :, s["back_off"]].int()] * scales[s["back_page"]][:, :, None]).to(x.dtype)


def _dense(s, codes, scales):
    """Keys or values of all sequences, padded: [B][heads][tokens][dim]."""
    c, table = s["case"], s["table"].long().clamp(min=0)
    x = s["values"][codes[table].int()]                         # [B][pages][heads][page][dim]
    x *= scales[table][:, :, :, None, None]
    return x.transpose(1, 2).reshape(c["B"], c["heads"], -1, c["dim"])


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "write":
        k, v = _write_plain(s, s["k"], s["k_codes"], s["k_scales"]), _write_plain(s, s["v"], s["v_codes"], s["v_scales"])
        return {"k": k, "v": v, "k_scales": s["k_scales"], "v_scales": s["v_scales"]}
    if c["kind"] == "read":
        page, off = s["table"].long()[s["seq"], s["pos"] // c["page"]], s["pos"] % c["page"]
        read = lambda codes, scales: (s["values"][codes[page, :, off].int()] * scales[page][:, :, None]).to(s["k"].dtype)  # noqa: E731
        return {"k": read(s["k_codes"], s["k_scales"]), "v": read(s["v_codes"], s["v_scales"])}
    B, H, D, group, most = c["B"], c["heads"], c["dim"], c["group"], max(_lengths(c)[0])
    q = torch.zeros((B, most, H, group, D), device=_DEV)
    q[s["seq"], s["nth"]] = s["q"].float().view(s["T"], H, group, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(B, H, group * most, D)
    x = q @ _dense(s, s["k_codes"], s["k_scales"]).transpose(2, 3)
    x *= D ** -0.5
    x = x.view(B, H, group, most, -1)
    key = torch.arange(x.shape[-1], device=_DEV)[None, None, :]
    fresh = (s["starts"][1:] - s["starts"][:-1])[:, None, None]
    pos = s["lens"][:, None, None] - fresh + torch.arange(most, device=_DEV)[None, :, None]
    hidden = key >= s["lens"][:, None, None]
    if c["causal"]:
        hidden = hidden | (key > pos)
    if c["window"]:
        hidden = hidden | (key <= pos - c["window"])
    x.masked_fill_(hidden[:, None, None], -math.inf)
    x -= x.amax(dim=-1, keepdim=True).clamp(min=-3e38)
    x.exp_()
    total = x.sum(dim=-1, keepdim=True)
    y = x.view(B, H, group * most, -1) @ _dense(s, s["v_codes"], s["v_scales"])
    y = y.view(B, H, group, most, D) / total
    return y.permute(0, 3, 1, 2, 4)[s["seq"], s["nth"]].reshape(s["T"], H * group, D).to(s["q"].dtype)


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_values():
    """Value of each code from the format's definition, one code after the other."""
    out = []
    for code in range(256):
        c = code & 127
        bits = format(c, "07b")
        lead = len(bits) - len(bits.lstrip("1"))
        rest = bits[lead + 1:]
        if lead == 0:
            v = c / 64
        elif lead == 7:
            v = 64.0
        else:
            v = 2.0 ** (lead - 1) * (1 + (int(rest, 2) / 2 ** len(rest) if rest else 0.0))
        out.append(-v if code >> 7 else v)
    return torch.tensor(out, dtype=torch.float64, device=_DEV)


def _nearest(x, values):
    """The value of the nearest code, the even code on a tie."""
    table = values[:128].contiguous()
    mag = x.abs().clamp(max=64.0).contiguous()
    hi = torch.searchsorted(table, mag).clamp(1, 127)
    below, above = mag - table[hi - 1], table[hi] - mag
    pick = torch.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, hi - 1)
    return torch.where(x < 0, -table[pick], table[pick])


def _exact_write(s, x, codes, scales, values):
    c, page = s["case"], s["case"]["page"]
    news, lens = _lengths(c)
    scales, back, at = scales.double().clone(), [], 0
    for b, (n, ln) in enumerate(zip(news, lens)):
        mine, p0 = x[at:at + n].double(), ln - n
        at += n
        for j in range(p0 // page, (ln - 1) // page + 1):
            p, lo, hi = int(s["table"][b, j]), max(p0, j * page), min(ln, (j + 1) * page)
            fresh = mine[lo - p0:hi - p0].transpose(0, 1)       # [heads][tokens][dim]
            held = values[codes[p, :, :lo - j * page].long()]
            amax = fresh.abs().amax(dim=(1, 2))
            need = torch.where(amax > 0, torch.exp2(torch.ceil(torch.log2(amax) - 1e-12) - _TOP), torch.zeros_like(amax))
            old = scales[p] if lo > j * page else torch.zeros_like(need)
            new = torch.maximum(old, need)
            grown = (new > old)[:, None, None]
            part = (old / new)[:, None, None]
            held = torch.where(grown, _nearest(held * part, values), held) * new[:, None, None]
            scales[p] = new
            back.append(torch.cat([held, _nearest(fresh / new[:, None, None], values) * new[:, None, None]], dim=1).transpose(0, 1))
    return torch.cat(back), scales


def exact(case, seed):
    s = prepare(case, seed)
    values, page = _exact_values(), case["page"]
    news, lens = _lengths(case)
    if case["kind"] == "write":
        k, ks = _exact_write(s, s["k"], s["k_codes"], s["k_scales"], values)
        v, vs = _exact_write(s, s["v"], s["v_codes"], s["v_scales"], values)
        return {"k": k, "v": v, "k_scales": ks, "v_scales": vs}

    def whole(b, codes, scales):
        """All tokens of sequence b: [heads][tokens][dim]."""
        p = s["table"][b, :-(-lens[b] // page)].long()
        x = values[codes[p].long()] * scales[p].double()[:, :, None, None]
        return x.transpose(0, 1).reshape(case["heads"], -1, case["dim"])[:, :lens[b]]

    if case["kind"] == "read":
        both = [torch.cat([whole(b, *pool)[:, ln - n:].transpose(0, 1) for b, (n, ln) in enumerate(zip(news, lens))])
                for pool in ((s["k_codes"], s["k_scales"]), (s["v_codes"], s["v_scales"]))]
        return {"k": both[0], "v": both[1]}
    out, at, group = torch.zeros(s["q"].shape, dtype=torch.float64, device=_DEV), 0, case["group"]
    for b, (n, ln) in enumerate(zip(news, lens)):
        k, v = whole(b, s["k_codes"], s["k_scales"]), whole(b, s["v_codes"], s["v_scales"])
        i, j = torch.arange(ln - n, ln, device=_DEV)[:, None], torch.arange(ln, device=_DEV)[None, :]
        seen = torch.ones((n, ln), dtype=torch.bool, device=_DEV)
        if case["causal"]:
            seen &= j <= i
        if case["window"]:
            seen &= j > i - case["window"]
        for h in range(case["heads"] * group):
            w = torch.einsum("td,sd->ts", s["q"][at:at + n, h].double(), k[h // group]) / math.sqrt(case["dim"])
            w = torch.softmax(w.masked_fill(~seen, -math.inf), dim=1)
            out[at:at + n, h] = w @ v[h // group]
        at += n
    return out
