"""The layer operators in 64 bits on the CPU, written from their definitions, and inputs for their tests."""
import math

import torch

from paper_2507_07145_amd import layer

DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn


def gen(seed):
    return torch.Generator().manual_seed(seed)


def values(codes):
    """e4m3 codes (uint8) as fp64."""
    return codes.cpu().view(E4M3).double()


def round_e4m3(x):
    """fp64 numbers of magnitude up to 464 as e4m3 values, ties to even (steps of 2^(e - 3), never less than 2^-9)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return (x / step).round() * step


def least_exponent(amax, lo, hi):
    """The least e in [lo, hi] with amax <= 448 2^e, by trying (amax: a float)."""
    e = lo
    while e < hi and amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def rows8(y):
    """(values in units of the scale before they are rounded, exponents) of fp64 rows, blocks of 128 columns."""
    M, N = y.shape
    nb = -(-N // 128)
    units, exps = torch.empty_like(y), torch.empty(M, nb, dtype=torch.int64)
    for m in range(M):
        for b in range(nb):
            block = y[m, b * 128:(b + 1) * 128]
            exps[m, b] = least_exponent(float(block.abs().max()), -126, 120)
            units[m, b * 128:(b + 1) * 128] = block * 2.0 ** -float(exps[m, b])
    return units, exps


def rotate(x, table, interleaved):
    """x fp64 [T][H][D], table fp64 [T][dims]."""
    dims = table.shape[1]
    half = dims // 2
    i = torch.arange(half)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = table[:, None, :half], table[:, None, half:]
    out = x.clone()
    out[..., first] = x[..., first] * c - x[..., second] * s
    out[..., second] = x[..., second] * c + x[..., first] * s
    return out


class Sequences:
    """Sequences with (new tokens, length with them) pairs on pages in random order; unused table entries are -1."""

    def __init__(self, pairs, page_tokens, seed=0, spare=2, max_len=None, width=None):
        self.pairs, self.P = pairs, page_tokens
        need = [-(-length // page_tokens) for _, length in pairs]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=gen(seed))
        width = max(need + [1]) if width is None else width
        self.table = torch.full((len(pairs), width), -1, dtype=torch.int32)
        at = 0
        for b, c in enumerate(need):
            self.table[b, :c] = order[at:at + c].to(torch.int32)
            at += c
        self.offsets = torch.tensor([0] + [n for n, _ in pairs]).cumsum(0).to(torch.int32)
        self.lens = torch.tensor([length for _, length in pairs], dtype=torch.int32)
        self.T = int(self.offsets[-1])
        self.max_new = max([n for n, _ in pairs] + [0])
        self.max_len = max([length for _, length in pairs] + [0]) if max_len is None else max_len

    def batch(self):
        self.held = [t.to(DEV) for t in (self.offsets, self.lens, self.table)]
        return layer.Batch(*self.held, tokens=self.T, max_new=self.max_new, max_len=self.max_len)


def random_cache(seq, heads, D, seed, garbage=0x7F, spread=2):
    """Cache contents on the CPU: random values and scales in written slots, `garbage` bytes elsewhere."""
    g = gen(seed)
    k = torch.randn(seq.pages, heads, seq.P, D, generator=g).clamp(-4, 4).to(E4M3).view(torch.uint8)
    v = torch.randn(seq.pages, heads, D, seq.P, generator=g).clamp(-4, 4).to(E4M3).view(torch.uint8)
    written = torch.zeros(seq.pages, seq.P, dtype=torch.bool)
    for b, (_, length) in enumerate(seq.pairs):
        for w in range(-(-length // seq.P)):
            written[seq.table[b, w], :min(seq.P, length - w * seq.P)] = True
    k[~written[:, None, :, None].expand_as(k)] = garbage
    v[~written[:, None, None, :].expand_as(v)] = garbage
    ks, vs = (torch.randint(127 - spread, 128 + spread, (seq.pages, heads), generator=g).to(torch.uint8) for _ in range(2))
    return k, v, ks, vs


def to_device(cache):
    return layer.Cache8(*[t.to(DEV) for t in cache])


def attend(seq, cache, q, scale, window=0, causal=True):
    """(out, what its error is measured by) in fp64: [T][Hq][D] each; the latter is the sum of weights times |v|, times the errors of
    the weights.  Those are: fp16 (2^-11), the scores' sums of D products in fp32 (D 2^-24 of the sum of the magnitudes, in the row's weight and in
    its total), exp2 (2^-20).  Beside them fp16's smallest step: 2^-25 of the row's largest weight (taken times the scale of v's page) for every
    token."""
    k, v, ks, vs = cache
    Hkv = k.shape[1]
    T, Hq, D = q.shape
    out, size = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    t = 0
    for b, (n, length) in enumerate(seq.pairs):
        slots = [(int(seq.table[b, j // seq.P]), j % seq.P) for j in range(length)]
        there = torch.tensor([0 <= p < seq.pages for p, _ in slots], dtype=torch.bool)
        pg = torch.tensor([p if 0 <= p < seq.pages else 0 for p, _ in slots], dtype=torch.long)
        sl = torch.tensor([s for _, s in slots], dtype=torch.long)
        for h in range(Hkv):
            kk = values(k[pg, h, sl]) * torch.exp2(ks[pg, h].double() - 127)[:, None]
            vv = values(v[pg, h, :, sl]) * torch.exp2(vs[pg, h].double() - 127)[:, None]
            for i in range(n):
                p = length - n + i
                seen = there.clone()
                j = torch.arange(length)
                if causal:
                    seen &= j <= p
                if window:
                    seen &= j > p - window
                if not bool(seen.any()):
                    continue
                for x in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    row = q[t + i, x].double()
                    w = torch.softmax(scale * (kk[seen] @ row), 0)
                    top = float((scale * (kk[seen].abs() @ row.abs())).max())
                    out[t + i, x] = w @ vv[seen]
                    scales = torch.exp2(vs[pg, h].double() - 127)[seen]
                    size[t + i, x] = (w @ vv[seen].abs()) * (2.0 ** -11 + 2.0 ** -20 + 2 * D * 2.0 ** -24 * top)
                    size[t + i, x] += 2.0 ** -25 * float((w * scales).max()) * (vv[seen].abs() / scales[:, None]).sum(0)
        t += n
    return out, size


def attend_limit(out, size):
    """bf16 rounding is up to 2^-8 of the value."""
    return 2.0 ** -7.98 * out.abs() + size + 1e-30
