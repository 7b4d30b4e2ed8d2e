"""Plain 64-bit forms of the key-value cache's operators, and batches to try them on.

Everything runs on the CPU from the definitions in include/dybit.h; the values of the codes come from the oracle's table."""
import math

import torch

from oracle import dybit_oracle as orc

def values():
    return torch.from_numpy(orc.decode_table(8, True)).double()


def half_step(t):
    """Half the distance of neighbouring codes around |t|, in units of the scale: 1/64 below 1, 2^(2e - 5) from 2^e on."""
    t = t.abs().clamp(max=63.0)
    return 0.5 * torch.where(t < 1, torch.full_like(t, 2.0 ** -6), torch.exp2(2 * torch.floor(torch.log2(t.clamp(min=1))) - 5))


def encode(x):
    """Codes of float64 numbers at scale 1: nearest value, ties to the even code; NaN gives 0."""
    table = values()[:128].contiguous()
    mag = torch.nan_to_num(x, nan=0.0, posinf=64.0, neginf=-64.0).abs().clamp(max=64.0).contiguous()
    hi = torch.searchsorted(table, mag).clamp(1, 127)
    below, above = mag - table[hi - 1], table[hi] - mag
    code = torch.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, hi - 1)
    return torch.where((x < 0) & (code > 0), code + 128, code).to(torch.uint8)


def needed_scale(x, top):
    """Scale that a block of float64 numbers asks for."""
    x = x[torch.isfinite(x)]
    amax = float(x.abs().max()) if x.numel() else 0.0
    if amax == 0.0:
        return 0.0
    mant, e = math.frexp(amax)
    e = e - 1 if mant == 0.5 else e
    return 2.0 ** max(-126, min(126, e - top))


class Batch:
    """Sequences of `lengths` tokens with `news` new ones, on pages of a pool in random order."""

    def __init__(self, lengths, news, page, heads, dim, seed=0, gap=0, spare=2, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.news, self.page, self.heads, self.dim, self.g = list(lengths), list(news), page, heads, dim, g
        used = [-(-n // page) for n in lengths]
        self.pages = sum(used) + spare
        self.most = max(max(used), 1) if max_pages is None else max_pages
        order = torch.randperm(self.pages, generator=g).to(torch.int32)
        self.table = torch.full((len(used), self.most), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(used):
            self.table[b, :n] = order[at:at + n]
            at += n
        starts = [gap]
        for n in news:
            starts.append(starts[-1] + n)
        self.starts, self.T = starts, starts[-1] + gap

    def rows(self, b):
        return range(self.starts[b], self.starts[b + 1])

    def position(self, b, row):
        return self.lengths[b] - self.news[b] + row - self.starts[b]

    def to(self, dev):
        return (self.table.to(dev), torch.tensor(self.starts, dtype=torch.int32, device=dev), torch.tensor(self.lengths, dtype=torch.int32, device=dev))

    def pool(self, spread=0.0):
        """Codes and scales of a pool in use; scales of neighbouring pages differ by up to 2^+-spread."""
        codes = torch.randint(0, 256, (self.pages, self.heads, self.page, self.dim), generator=self.g).to(torch.uint8)
        codes = torch.where(torch.rand(codes.shape, generator=self.g) < 0.7, codes & 0xbf, codes)      # most below 1
        e = torch.round((2 * torch.rand((self.pages, self.heads), generator=self.g) - 1) * spread)
        return codes, torch.exp2(e - 1).float()


def write(batch, x, codes, scales, top):
    """What a write makes of (codes, scales): x [T][heads][dim]."""
    codes, scales, x = codes.clone(), scales.clone().double(), x.double()
    for b, n in enumerate(batch.news):
        groups = {}
        for row in batch.rows(b):
            pos = batch.position(b, row)
            if pos >= 0:
                groups.setdefault(pos // batch.page, []).append((pos % batch.page, row))
        for j, tokens in groups.items():
            p = int(batch.table[b, j])
            if not 0 <= p < batch.pages:
                continue
            first = tokens[0][0]
            for h in range(batch.heads):
                fresh = torch.stack([x[row, h] for _, row in tokens])
                need, old = needed_scale(fresh, top), float(scales[p, h]) if first > 0 else 0.0
                s = max(need, old)
                if s > old and first > 0:
                    held = values()[codes[p, h, :first].long()] * (old / s)
                    codes[p, h, :first] = encode(held)
                for (off, _), v in zip(tokens, fresh):
                    codes[p, h, off] = encode(v / s) if s > 0 else 0
                scales[p, h] = s
    return codes, scales.float()


def read(batch, codes, scales):
    """[T][heads][dim] in 64 bits and the rows that belong to a sequence."""
    out, mine = torch.zeros((batch.T, batch.heads, batch.dim), dtype=torch.float64), torch.zeros(batch.T, dtype=torch.bool)
    for b in range(len(batch.news)):
        for row in batch.rows(b):
            mine[row] = True
            pos = batch.position(b, row)
            if pos < 0:
                continue
            p = int(batch.table[b, pos // batch.page])
            if 0 <= p < batch.pages:
                out[row] = values()[codes[p, :, pos % batch.page].long()] * scales[p].double()[:, None]
    return out, mine


def attention(batch, q, k_pool, v_pool, scale, causal=True, window=0):
    """(y, lse, bound of |y - kernel's| without its own rounding, rows that belong to a sequence).

    The bound, per element, with the probabilities w_j (sum 1) and S = sum_j w_j |v_j|:
      f16 probabilities   2^-11 S, and 2^-25 of the largest |v| for each key where they are subnormal
      scores              q . k adds D products in fp32 whose additions may cut off: off by D 2^-23 sum |q k| at most, times
                          the scale; the product with the scale, the maximum's subtraction and 2^x are off by 4 steps 2^-24
                          of the largest |x| in base 2 and 2^-22 of the probability.  A score off by d moves y by 2 d S
      sums                fp32, n additions that may cut off: 2 n 2^-23 S"""
    T, Hq, D = q.shape
    group = Hq // batch.heads
    y, lse = torch.zeros((T, Hq, D), dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64)
    bound, mine = torch.zeros_like(y), torch.zeros(T, dtype=torch.bool)
    for b, n in enumerate(batch.news):
        ln = batch.lengths[b]
        rows = list(batch.rows(b))
        mine[rows] = True
        if n == 0 or ln == 0:
            continue
        entries = batch.table[b, :-(-ln // batch.page)].long()
        there = (entries >= 0) & (entries < batch.pages)
        dense = []
        for codes, scales in (k_pool, v_pool):
            x = values()[codes[entries.clamp(0, batch.pages - 1)].long()] * scales[entries.clamp(0, batch.pages - 1)].double()[:, :, None, None]
            dense.append(x.transpose(1, 2).reshape(-1, batch.heads, D)[:ln])
        k, v = dense
        seen_page = there.repeat_interleave(batch.page)[:ln]
        pos = torch.tensor([batch.position(b, r) for r in rows])[:, None]
        key = torch.arange(ln)[None, :]
        seen = seen_page[None, :].expand(n, ln).clone()
        if causal:
            seen &= key <= pos
        if window:
            seen &= key > pos - window
        for h in range(Hq):
            kh, vh, qh = k[:, h // group], v[:, h // group], q[rows, h].double()
            x = (qh @ kh.t()) * scale
            x = x.masked_fill(~seen, -math.inf)
            any_ = seen.any(dim=1)
            w = torch.softmax(x, dim=1).masked_fill(~any_[:, None], 0.0).nan_to_num(0.0) if bool(torch.isfinite(qh).all()) else \
                torch.softmax(x, dim=1).masked_fill(~any_[:, None], 0.0)
            y[rows, h] = w @ vh
            lse[rows, h] = torch.logsumexp(x, dim=1)
            S = w @ vh.abs()
            big = (qh.abs() @ kh.abs().t()).masked_fill(~seen, 0.0).amax(dim=1, keepdim=True) * scale
            off = D * 2.0 ** -23 * big + 4 * 2.0 ** -24 * 1.4427 * (big + 16) + 2.0 ** -22
            vmax = torch.where(seen.any(dim=0)[:, None], vh.abs(), torch.zeros_like(vh)).amax()
            bound[rows, h] = (2.0 ** -11 + 2 * off + 2 * ln * 2.0 ** -23) * S + ln * 2.0 ** -25 * vmax * (w.amax(dim=1, keepdim=True))
    return y, lse, bound, mine


def step(dtype):
    """Half a step of a type, relative to the value."""
    return torch.finfo(dtype).eps / 2


def check_attention(got, got_lse, want, dtype, name=""):
    y, lse, bound, mine = want
    err = (got.double().cpu() - y).abs()[mine]
    room = (bound + step(dtype) * (y.abs() + bound) + torch.finfo(dtype).smallest_normal * 2.0 ** -10)[mine]
    assert bool((err <= room).all()), (name, float((err / room.clamp(min=1e-300)).max()))
    if got_lse is not None:
        a, b = got_lse.double().cpu()[mine], lse[mine]
        empty = b == -math.inf
        assert bool((a[empty] == -math.inf).all()), name
        assert bool(((a - b)[~empty].abs() <= 2.0 ** -16 * (1 + b[~empty].abs())).all()), (name, float((a - b)[~empty].abs().max()))
