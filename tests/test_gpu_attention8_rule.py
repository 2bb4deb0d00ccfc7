"""Calls that the rule itself gives to the attention's kernel for many rows: several sequences, many tiles of rows, against 64 bits."""
import ctypes

import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


def _attend(seq, cache, q, scale, window, causal):
    """r.attend, all rows of a sequence and head at once."""
    k, v, ks, vs = cache
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    g = Hq // Hkv
    out, size = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    t = 0
    for b, (n, length) in enumerate(seq.pairs):
        if n == 0:
            continue
        pg = torch.stack([seq.table[b, j // seq.P] for j in range(length)]).long()
        sl = torch.arange(length) % seq.P
        there = (pg >= 0) & (pg < seq.pages)
        pg = pg.where(there, torch.zeros_like(pg))
        p, j = torch.arange(length - n, length)[:, None], torch.arange(length)[None]
        seen = there[None].expand(n, length).clone()
        if causal:
            seen &= j <= p
        if window:
            seen &= j > p - window
        seen = seen.repeat_interleave(g, 0)
        for h in range(Hkv):
            scales = torch.exp2(vs[pg, h].double() - 127)[:, None]
            kk, units = r.values(k[pg, h, sl]) * torch.exp2(ks[pg, h].double() - 127)[:, None], r.values(v[pg, h, :, sl])
            kk[~there], units[~there] = 0, 0
            rows = q[t:t + n, h * g:(h + 1) * g].double().reshape(n * g, D)
            w = (scale * rows @ kk.t()).masked_fill(~seen, float("-inf")).softmax(1).nan_to_num(0.0)
            top = (scale * rows.abs() @ kk.abs().t()).where(seen, torch.zeros(())).amax(1, keepdim=True)
            o, z = w @ (units * scales), (w @ (units * scales).abs()) * (2.0 ** -11 + 2.0 ** -20 + 2 * D * 2.0 ** -24 * top)
            z += 2.0 ** -25 * (w * scales.t()).amax(1, keepdim=True) * (seen.double() @ units.abs())
            out[t:t + n, h * g:(h + 1) * g], size[t:t + n, h * g:(h + 1) * g] = o.view(n, g, D), z.view(n, g, D)
        t += n
    return out, size


def _workspace(cache, batch, q, window, causal):
    a = layer.ccq_attn(q.shape[1], int(causal), window, q.shape[2] ** -0.5)
    return layer._load().ccq_attention_workspace_bytes(ctypes.byref(cache.desc), ctypes.byref(batch.desc), ctypes.byref(a))


@pytest.mark.parametrize("pairs,P,Hkv,Hq,window,causal", [
    ([(512, 1300), (448, 900)], 64, 4, 32, 0, True), ([(800, 1500), (1, 700), (300, 300), (0, 200)], 16, 4, 32, 900, True), ([(512, 1100)], 128, 8, 64, 0, False),
    ([(700, 700), (650, 2000)], 32, 4, 28, 0, True),
])
def test_many_rows_by_the_rule(pairs, P, Hkv, Hq, window, causal):
    seq = r.Sequences(pairs, P, 5)
    held = r.random_cache(seq, Hkv, 128, 6)
    seq.table[0, 3] = -1   # a page that is not there
    cache, batch = r.to_device(held), seq.batch()
    q = torch.randn(seq.T, Hq, 128, generator=r.gen(8)).bfloat16()
    image = 4 * 64 * 128
    assert _workspace(cache, batch, q, window, causal) >= len(pairs) * Hkv * (min(seq.max_len, window + seq.max_new if window else seq.max_len) // 64) * image
    got = layer.attention(cache, batch, q.to(r.DEV), window=window, causal=causal)
    want, size = _attend(seq, held, q, 128 ** -0.5, window, causal)
    assert bool(((got.cpu().double() - want).abs() <= r.attend_limit(want, size)).all())
    assert torch.equal(layer.attention(cache, batch, q.to(r.DEV), window=window, causal=causal), got)


def test_the_reference_is_the_other_one():
    seq = r.Sequences([(9, 70), (1, 40)], 16, 1)
    held = r.random_cache(seq, 2, 64, 2)
    seq.table[0, 1] = -1
    q = torch.randn(seq.T, 4, 64, generator=r.gen(3)).bfloat16()
    for window, causal in ((0, True), (20, True), (0, False)):
        for mine, other in zip(_attend(seq, held, q, 0.125, window, causal), r.attend(seq, held, q, 0.125, window, causal)):
            assert torch.allclose(mine, other, rtol=1e-9, atol=1e-12)
