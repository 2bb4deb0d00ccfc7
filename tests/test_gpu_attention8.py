"""attention over the 8-bit cache against 64 bits: decode and prompts, ragged lengths, windows, page sizes, heads, garbage in what is not seen."""
import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


def _run(pairs, P, D, Hkv, Hq, window=0, causal=True, seed=0, scale=None, garbage=0x7F, spread=2, q=None, mutate=None, **kw):
    seq = r.Sequences(pairs, P, seed, **kw)
    cache = r.random_cache(seq, Hkv, D, seed + 1, garbage, spread)
    if q is None:
        q = torch.randn(seq.T, Hq, D, generator=r.gen(seed + 2)).bfloat16()
    if mutate is not None:
        mutate(seq, cache, q)
    scale = D ** -0.5 if scale is None else scale
    got = layer.attention(r.to_device(cache), seq.batch(), q.to(r.DEV), scale=scale, window=window, causal=causal)
    want, size = r.attend(seq, cache, q, scale, window, causal)
    got = got.cpu().double()
    assert bool(((got - want).abs() <= r.attend_limit(want, size)).all()), float(((got - want).abs() / (r.attend_limit(want, size))).max())
    return got


DECODE = [
    ([(1, 1)], 16, 64, 1, 1), ([(1, 15), (1, 16), (1, 17), (1, 63), (1, 64), (1, 65)], 16, 64, 2, 4), ([(1, 200), (1, 3), (1, 0), (1, 130)], 32, 128, 2, 14),
    ([(1, 5000)], 64, 128, 1, 8), ([(1, 3000), (1, 1), (1, 511)], 128, 128, 2, 2), ([(1, 1025)], 256, 64, 1, 16), ([(1, 700)], 64, 128, 1, 32), ([(1, 300)], 64, 64, 1, 40),
    ([(0, 50), (1, 50)], 64, 128, 1, 5),
]


@pytest.mark.parametrize("pairs,P,D,Hkv,Hq", DECODE)
@pytest.mark.parametrize("window", [0, 1, 100])
def test_decode(pairs, P, D, Hkv, Hq, window):
    _run(pairs, P, D, Hkv, Hq, window, seed=P + Hq)


PROMPT = [
    ([(2, 2)], 16, 64, 1, 1), ([(3, 70), (5, 5), (1, 40), (0, 9)], 16, 128, 2, 6), ([(16, 300)], 64, 128, 1, 2), ([(33, 33), (17, 100)], 32, 64, 2, 2),
    ([(70, 70)], 64, 128, 1, 7), ([(130, 400), (64, 64), (9, 1000)], 64, 128, 1, 4), ([(200, 333)], 128, 64, 2, 8), ([(300, 300)], 16, 128, 1, 1), ([(140, 650)], 256, 128, 1, 5),
]


@pytest.mark.parametrize("pairs,P,D,Hkv,Hq", PROMPT)
@pytest.mark.parametrize("window,causal", [(0, True), (50, True), (0, False)])
def test_prompt(pairs, P, D, Hkv, Hq, window, causal):
    _run(pairs, P, D, Hkv, Hq, window, causal, seed=P + Hq)


@pytest.mark.parametrize("pairs,Hq", [([(1, 600)], 4), ([(40, 300)], 3), ([(80, 300)], 3)])
def test_scales_far_apart(pairs, Hq):
    """Pages whose scales differ by up to 2^60: weights and values of each keep their precision next to the others."""
    _run(pairs, 16, 64, 1, Hq, seed=3, spread=6)
    def mutate(seq, cache, q):
        cache[2][:] = 127
        cache[3][:] = torch.randint(127 - 30, 127 + 31, cache[3].shape, generator=r.gen(9)).to(torch.uint8)
    _run(pairs, 16, 64, 1, Hq, seed=4, mutate=mutate)


@pytest.mark.parametrize("pairs,Hq", [([(1, 900)], 8), ([(50, 400)], 2), ([(100, 400)], 2)])
def test_peaked_rows(pairs, Hq):
    """Large scores: one token takes all the weight, wherever it lies."""
    _run(pairs, 32, 128, 1, Hq, seed=7, scale=2.0)


@pytest.mark.parametrize("pairs", [[(1, 200), (1, 90)], [(20, 200), (8, 90)], [(90, 200), (70, 90)]])
def test_pages_that_are_not_there(pairs):
    """Tokens of such pages are left out; a row that sees no other is zero."""
    def mutate(seq, cache, q):
        seq.table[0, 1], seq.table[0, 5] = -1, 1 << 30
        seq.table[1, :] = -7
    got = _run(pairs, 32, 64, 2, 4, seed=2, mutate=mutate)
    assert not bool(got[pairs[0][0]:].any())
    # with a window: pages before it may be gone, or belong to others and hold anything
    def gone(seq, cache, q):
        seq.table[0, 0] = -1
        cache[0][seq.table[0, 1]], cache[1][seq.table[0, 1]] = 0x7F, 0xFF
    _run([(5, 200)], 32, 64, 2, 4, window=100, seed=2, mutate=gone)


def test_nan_in_queries_and_keys_reach_the_rows_that_see_them():
    pairs, P, D = [(30, 80)], 16, 64
    seq = r.Sequences(pairs, P, 1)
    for rows in (1, 4):
        cache = r.random_cache(seq, 1, D, 2)
        q = torch.randn(30, rows, D, generator=r.gen(3)).bfloat16()
        q[11, 0, 5] = float("nan")
        page, slot = int(seq.table[0, 70 // P]), 70 % P   # position 70: new token 20
        cache[0][page, 0, slot, 3] = 0x7F
        got = layer.attention(r.to_device(cache), seq.batch(), q.to(r.DEV)).cpu()
        nan = got.isnan().all(2)
        want = torch.zeros(30, rows, dtype=torch.bool)
        want[20:] = True
        want[11, 0] = True
        assert torch.equal(nan, want) and torch.equal(got.isnan().any(2), want)


def test_lengths_past_the_bounds_and_the_table():
    """Cached tokens past max_len or the table are left out; tokens past max_new keep their rows."""
    seq = r.Sequences([(1, 100)], 16, 0)
    cache = r.random_cache(seq, 1, 64, 1)
    q = torch.randn(1, 2, 64, generator=r.gen(2)).bfloat16()
    for max_len, width in ((40, 7), (100, 3), (64, 7)):
        table = seq.table[:, :width].contiguous().to(r.DEV)
        batch = layer.Batch(seq.offsets.to(r.DEV), seq.lens.to(r.DEV), table, tokens=1, max_new=1, max_len=max_len)
        got = layer.attention(r.to_device(cache), batch, q.to(r.DEV)).cpu().double()
        cut = r.Sequences([(1, min(max_len, 16 * width))], 16, 0)
        cut.table, cut.pages = seq.table, seq.pages
        want, size = r.attend(cut, cache, q, 64 ** -0.5)
        assert bool(((got - want).abs() <= r.attend_limit(want, size)).all())
    q = torch.randn(6, 2, 64, generator=r.gen(3)).bfloat16().to(r.DEV)
    batch = layer.Batch(torch.tensor([0, 6], dtype=torch.int32).to(r.DEV), seq.lens.to(r.DEV), seq.table.to(r.DEV), tokens=6, max_new=4, max_len=100)
    out = torch.full((6, 2, 64), 7.0, dtype=torch.bfloat16, device=r.DEV)
    layer.attention(r.to_device(cache), batch, q, out=out)
    assert bool((out[4:] == 7).all()) and not bool((out[:4] == 7).any())


def test_strides_and_the_general_path():
    """Queries and results as slices of wider tensors, a workspace of the caller's, another stream: the same bits."""
    pairs, P, D, Hkv, Hq = [(3, 2000), (1, 700)], 64, 128, 2, 8
    seq = r.Sequences(pairs, P, 5)
    cache = r.to_device(r.random_cache(seq, Hkv, D, 6))
    wide = torch.randn(seq.T, Hq + 4, D + 8, generator=r.gen(7)).bfloat16().to(r.DEV)
    q = wide[:, 2:2 + Hq, :D]
    want = layer.attention(cache, seq.batch(), q.contiguous())
    out = torch.full((seq.T, Hq + 1, D + 16), 7.0, dtype=torch.bfloat16, device=r.DEV)
    layer.attention(cache, seq.batch(), q, out=out[:, :Hq, :D], workspace=torch.empty(64 << 20, dtype=torch.uint8, device=r.DEV))
    assert torch.equal(out[:, :Hq, :D], want)
    assert bool((out[:, Hq:] == 7).all()) and bool((out[:, :, D:] == 7).all())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = layer.attention(cache, seq.batch(), q, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_a_batch_of_nothing():
    seq = r.Sequences([(0, 5), (0, 0)], 16, 0)
    c = r.to_device(r.random_cache(r.Sequences([(0, 5), (0, 1)], 16, 0), 1, 64, 1))
    assert layer.attention(c, seq.batch(), torch.empty(0, 2, 64, dtype=torch.bfloat16, device=r.DEV)).shape == (0, 2, 64)


def test_offsets_past_32_bits():
    """A cache of more than 4 GiB of keys: the last pages' tokens are the right ones."""
    P, D, H = 256, 128, 8
    pages = (1 << 32) // (P * D * H) + 4
    c = layer.Cache8.empty(pages, P, H, D, r.DEV)
    seq = r.Sequences([(1, 600), (3, 300)], P, 0, spare=0)
    small = r.random_cache(seq, H, D, 1)
    where = torch.tensor([pages - 1 - i for i in range(seq.pages)])
    for mine, theirs in zip((c.k, c.v, c.k_scales, c.v_scales), small):
        mine[where.to(r.DEV)] = theirs.to(r.DEV)
    q = torch.randn(4, 16, D, generator=r.gen(2)).bfloat16()
    want, size = r.attend(seq, small, q, D ** -0.5)
    table = seq.table.clone()
    table[table >= 0] = where[table[table >= 0].long()].to(torch.int32)
    seq.table = table
    got = layer.attention(c, seq.batch(), q.to(r.DEV)).cpu().double()
    assert bool(((got - want).abs() <= r.attend_limit(want, size)).all())
    # and the append's
    k = torch.randn(4, H, D, generator=r.gen(3)).bfloat16()
    layer.cache_append(c, seq.batch(), k.to(r.DEV), k.to(r.DEV))
    page, slot = int(table[0, 599 // P]), 599 % P
    for held, s in ((r.values(c.k[page, :, slot].contiguous()), c.k_scales), (r.values(c.v[page, :, :, slot].contiguous()), c.v_scales)):
        x = held * torch.exp2(s[page].cpu().double() - 127)[:, None]
        assert bool(((x - k[0].double()).abs() <= k[0].double().abs() * 2.0 ** -4 + 2.0 ** -6).all())
