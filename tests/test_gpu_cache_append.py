"""cache_append and rope_table against 64 bits: page sizes, partly filled pages, growing scales, rotary layouts, NaN, pages that are not there."""
import math

import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


def _append(seq, cache, k, v, table, interleaved, positions=None):
    """The cache after the append in fp64: values in units of the scale before they are rounded (older tokens: as held, brought to the new
    scale), exponents, and which slots are new."""
    Hkv, D, P = k.shape[1], k.shape[2], seq.P
    kc, vc, ks, vs = cache
    units = [r.values(kc), r.values(vc).transpose(2, 3).contiguous()]
    exps = [ks.long() - 127, vs.long() - 127]
    new_slots = torch.zeros(seq.pages, P, dtype=torch.bool)
    t = 0
    for b, (n, length) in enumerate(seq.pairs):
        pos = torch.arange(length - n, length)
        kk = k[t:t + n].double()
        if table is not None:
            at = pos if positions is None else positions[t:t + n].long()
            kk = r.rotate(kk, table[at.clamp(0, table.shape[0] - 1)].double(), interleaved)
        vv = v[t:t + n].double()
        t += n
        bad = ~vv.isfinite().all(2)
        kk[bad], vv[bad] = float("nan"), 0.0
        for w in sorted(set((pos[pos >= 0] // P).tolist())):
            page = int(seq.table[b, w]) if w < seq.table.shape[1] else -1
            if not 0 <= page < seq.pages:
                continue
            here = (pos // P == w) & (pos >= 0)
            slots = pos[here] % P
            older = int(slots[0])
            new_slots[page, slots] = True
            for which, x in ((0, kk), (1, vv)):
                for h in range(Hkv):
                    x_h = x[here][:, h]
                    e = r.least_exponent(float(x_h[x_h.isfinite()].abs().max()) if bool(x_h.isfinite().any()) else 0.0, -60, 60)
                    if older:
                        e_old = int(exps[which][page, h])
                        e = max(e, e_old)
                        units[which][page, h, :older] = r.round_e4m3(units[which][page, h, :older] * 2.0 ** (e_old - e))
                    exps[which][page, h] = e
                    units[which][page, h, slots] = torch.where(x_h.isfinite(), (x_h * 2.0 ** -e).clamp(-448, 448), float("nan"))
    return units, exps, new_slots


def _check_cache(c, before, units, exps, new_slots):
    for codes, scales, u, e, was in ((c.k, c.k_scales, units[0], exps[0], before[0]), (c.v, c.v_scales, units[1], exps[1], before[1])):
        assert torch.equal(scales.cpu().long() - 127, e)
        got = r.values(codes)
        if codes is c.v:
            got, was = got.transpose(2, 3), was.transpose(2, 3)
        new = new_slots[:, None, :, None].expand_as(got)
        # new tokens: half a step (2^-4 of the value, 2^-10 below the smallest normal number), and 2^-22 for the rotation in fp32
        near = (got - u).abs() <= u.abs() * (2.0 ** -4 + 2.0 ** -18) + 2.0 ** -10 + 2.0 ** -14
        assert bool((near | (got.isnan() & u.isnan()))[new].all())
        # all others: exactly
        same = (got == u) | (got.isnan() & u.isnan())
        assert bool(same[~new].all())


def _case(pairs, P, D, Hkv, Hq, dims, interleaved, seed=0, kind=1.0, positions=False, **kw):
    seq = r.Sequences(pairs, P, seed, **kw)
    # the cache holds older tokens where the sequences' pages are
    held = r.Sequences(pairs, P, seed)
    k0, v0, ks, vs = r.random_cache(held, Hkv, D, seed + 1)
    for b, (n, length) in enumerate(pairs):   # slots from the first new one on are not written yet
        for w in range(-(-length // P)):
            page, first = int(seq.table[b, w]), max(0, length - n - w * P)
            k0[page, :, first:], v0[page, :, :, first:] = 0x7F, 0x7F
    before = (k0, v0, ks, vs)
    g = r.gen(seed + 2)
    k = (kind * torch.randn(seq.T, Hkv, D, generator=g)).bfloat16()
    v = (kind * torch.randn(seq.T, Hkv, D, generator=g)).bfloat16()
    q = torch.randn(seq.T, Hq, D, generator=g).bfloat16()
    table = None
    if dims:
        angle = torch.rand(seq.max_len + 3, dims // 2, generator=g) * 6.28
        table = torch.cat((angle.cos(), angle.sin()), 1)
    pos = torch.randint(0, seq.max_len + 3, (seq.T,), generator=g).to(torch.int32) if positions else None
    return seq, before, k, v, q, table, pos


CASES = [
    # pairs (new, length), page, dim, kv heads, q heads, rotated, interleaved
    ([(1, 1)], 16, 64, 1, 1, 64, False),
    ([(1, 17), (1, 16), (1, 33), (1, 100)], 16, 64, 2, 6, 64, True),
    ([(1, 8191), (1, 65), (1, 64), (1, 128)], 64, 128, 8, 64, 128, False),
    ([(5, 5), (3, 70), (16, 33), (0, 12), (1, 31)], 32, 128, 2, 10, 64, True),
    ([(300, 300), (77, 200)], 64, 128, 2, 14, 64, False),
    ([(300, 333)], 128, 64, 3, 3, 32, True),
    ([(513, 700), (2, 257)], 256, 128, 1, 8, 128, False),
    ([(260, 300)], 256, 64, 1, 2, 10, False),      # half of the rotated dimensions is no multiple of eight
    ([(40, 90)], 16, 128, 2, 2, 6, True),
    ([(9, 20)], 16, 128, 2, 2, 0, False),
]


@pytest.mark.parametrize("pairs,P,D,Hkv,Hq,dims,interleaved", CASES)
@pytest.mark.parametrize("kind,positions", [(1.0, False), (1e-3, True), (300.0, False)])
def test_append(pairs, P, D, Hkv, Hq, dims, interleaved, kind, positions):
    positions = positions and dims > 0
    seq, before, k, v, q, table, pos = _case(pairs, P, D, Hkv, Hq, dims, interleaved, seed=len(pairs) * 10 + P, kind=kind, positions=positions)
    c = r.to_device(before)
    rope = layer.Rope(table.to(r.DEV), interleaved=interleaved, positions=None if pos is None else pos.to(r.DEV)) if dims else None
    # keys, values and queries as slices of one product's output
    fused = torch.cat((q, k, v), 1).to(r.DEV)
    out = layer.cache_append(c, seq.batch(), fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:], q=fused[:, :Hq], rope=rope)
    _check_cache(c, before, *_append(seq, before, k, v, table, interleaved, pos))
    want = q.double()
    if dims:
        at = torch.cat([torch.arange(length - n, length) for n, length in pairs]) if pos is None else pos.long()
        want = r.rotate(want, table[at].double(), interleaved)
    size = q.double().abs() + q.double().abs().amax(2, keepdim=True)
    assert bool(((out.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -22 * size).all())
    # queries alone, in place
    before_q = c.k.clone()
    assert layer.cache_append(c, seq.batch(), None, None, q=fused[:, :Hq], q_out=fused[:, :Hq], rope=rope).data_ptr() == fused.data_ptr()
    assert torch.equal(fused[:, :Hq], out) and torch.equal(c.k, before_q)


def test_token_by_token_equals_growing_scales():
    """A page filled one token at a time, each larger than the last: every step's scale and bytes follow the definition."""
    P, D, H = 16, 64, 2
    cache = None
    for step in range(P + 2):
        pairs = [(1, step + 1)]
        seq = r.Sequences(pairs, P, 3, spare=0, max_len=P + 2)
        seq.pages, seq.table = 2, torch.tensor([[1, 0]], dtype=torch.int32)
        if cache is None:
            cache = [torch.full((2, H, P, D), 0x7F, dtype=torch.uint8), torch.full((2, H, D, P), 0x7F, dtype=torch.uint8), *torch.zeros(2, 2, H, dtype=torch.uint8)]
        g = r.gen(step)
        k, v = ((torch.randn(1, H, D, generator=g) * 1.5 ** (step % 7)).bfloat16() for _ in range(2))
        c = r.to_device(cache)
        assert layer.cache_append(c, seq.batch(), k.to(r.DEV), v.to(r.DEV)) is None
        _check_cache(c, cache, *_append(seq, cache, k, v, None, False))
        cache = [t.cpu() for t in (c.k, c.v, c.k_scales, c.v_scales)]


def test_nan_and_infinities():
    seq, before, k, v, _, _, _ = _case([(20, 40)], 16, 64, 2, 2, 0, False, seed=5)
    k[3, 0, 7], k[4, 1, 0], v[6, 1, 9], v[7, 0, 63] = float("nan"), float("inf"), float("-inf"), float("nan")
    c = r.to_device(before)
    layer.cache_append(c, seq.batch(), k.to(r.DEV), v.to(r.DEV))
    want = _append(seq, before, k, v, None, False)
    _check_cache(c, before, *want)
    assert not bool(r.values(c.v)[..., :][torch.zeros_like(r.values(c.v), dtype=torch.bool)].any())
    written = want[2]
    assert bool(r.values(c.v).transpose(2, 3)[written[:, None, :].expand(-1, 2, -1)].isfinite().all())


def test_zeros_and_tiny_and_huge():
    for x in (0.0, 1e-38, 2.0 ** -52, 1e20, 3e38):
        seq, before, k, v, _, _, _ = _case([(3, 3), (4, 20)], 16, 64, 1, 1, 0, False, seed=6)
        k, v = torch.full_like(k, x), torch.full_like(v, -x)
        c = r.to_device(before)
        layer.cache_append(c, seq.batch(), k.to(r.DEV), v.to(r.DEV))
        _check_cache(c, before, *_append(seq, before, k, v, None, False))


def test_pages_that_are_not_there_and_bounds_that_cut():
    """Entries of the table outside the cache, tokens past max_len, past the table and past max_new are left out; lengths shorter than the new tokens too."""
    seq, before, k, v, q, _, _ = _case([(40, 70), (10, 20)], 16, 64, 2, 2, 0, False, seed=8)
    seq.table[0, 2], seq.table[1, 1] = -1, 1 << 30
    c = r.to_device(before)
    layer.cache_append(c, seq.batch(), k.to(r.DEV), v.to(r.DEV))
    _check_cache(c, before, *_append(seq, before, k, v, None, False))
    # a length that is shorter than the new tokens: the first ones have no place
    offsets, lens = torch.tensor([0, 10], dtype=torch.int32).to(r.DEV), torch.tensor([4], dtype=torch.int32).to(r.DEV)
    table = torch.tensor([[1]], dtype=torch.int32).to(r.DEV)
    c = r.to_device(before)
    layer.cache_append(c, layer.Batch(offsets, lens, table, tokens=10, max_new=10, max_len=16), k[:10].to(r.DEV), v[:10].to(r.DEV))
    short = r.Sequences([(4, 4)], 16)
    short.pages, short.table = seq.pages, torch.tensor([[1]], dtype=torch.int32)
    _check_cache(c, before, *_append(short, before, k[6:10], v[6:10], None, False))
    for bound in (dict(max_new=10, max_len=20), dict(max_new=7, max_len=64), dict(max_new=10, max_len=64)):
        lens = torch.tensor([30], dtype=torch.int32).to(r.DEV)
        wide = torch.tensor([[1] if bound == dict(max_new=10, max_len=64) else [1, 2]], dtype=torch.int32).to(r.DEV)
        if bound == dict(max_new=10, max_len=64):
            lens = torch.tensor([17], dtype=torch.int32).to(r.DEV)   # the last of the new tokens is past a table of one page
        c = r.to_device(before)
        layer.cache_append(c, layer.Batch(offsets, lens, wide, tokens=10, **bound), k[:10].to(r.DEV), v[:10].to(r.DEV))
        first = int(lens[0]) - 10
        kept = min(bound["max_new"], bound["max_len"] - first if bound["max_len"] == 20 else 10, 16 * wide.shape[1] - first)
        cut = r.Sequences([(max(kept, 0), first + max(kept, 0))], 16)
        cut.pages, cut.table = seq.pages, wide.cpu()
        _check_cache(c, before, *_append(cut, before, k[:max(kept, 0)], v[:max(kept, 0)], None, False))


def _angles(dims, base, kind, factor, orig, fast, slow):
    i = torch.arange(dims // 2, dtype=torch.float64)
    f = base ** (-2 * i / dims)
    if kind == "linear":
        f = f / factor
    if kind == "base":
        f = (base * factor ** (dims / (dims - 2))) ** (-2 * i / dims)
    if kind == "parts":
        at = lambda turns: dims * math.log(orig / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), dims - 1)
        mix = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        f = f * (1 - mix) + f / factor * mix
    return f


@pytest.mark.parametrize("kind,factor,magnitude", [("none", 1.0, 1.0), ("linear", 4.0, 1.0), ("base", 8.0, 1.0), ("parts", 16.0, 1.277), ("parts", 1.0, 1.0)])
@pytest.mark.parametrize("rows,dims", [(1, 2), (777, 64), (70000, 128), (33, 10)])
def test_rope_table(kind, factor, magnitude, rows, dims):
    if kind == "base" and dims < 4:
        return
    got = layer.rope_table(rows, dims, base=500000.0, kind=kind, factor=factor, original_length=4096.0, magnitude=magnitude).cpu().double()
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * _angles(dims, 500000.0, kind, factor, 4096.0, 32.0, 1.0)
    want = torch.cat((angle.cos(), angle.sin()), 1) * magnitude
    # fp32 rounding, and angles of up to 70000 in 64 bits
    assert float((got - want).abs().max()) <= 2.0 ** -24 * magnitude + 1e-9
