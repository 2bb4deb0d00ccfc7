"""Attention beside pages that no row sees, missing or before the window: their scale bytes may hold anything, as their codes may."""
import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1], ids=["few", "many"], autouse=True)
def kernel(request):
    layer._load().ccq_attention_force(request.param)
    yield
    layer._load().ccq_attention_force(-1)


def _sequences(pairs, P, seed):
    """Page 0 belongs to no sequence."""
    seq = r.Sequences(pairs, P, seed)
    seq.table[seq.table >= 0] += 1
    seq.pages += 1
    return seq


def _check(seq, cache, q, window=0):
    got = layer.attention(r.to_device(cache), seq.batch(), q.to(r.DEV), window=window).cpu().double()
    want, size = r.attend(seq, cache, q, q.shape[2] ** -0.5, window)
    assert bool(((got - want).abs() <= r.attend_limit(want, size)).all())


BYTES = [(0, 127), (255, 127), (127, 0), (127, 255), (127, 254), (0, 255), (255, 0)]


@pytest.mark.parametrize("k_byte,v_byte", BYTES)
@pytest.mark.parametrize("pairs", [[(1, 300), (1, 130)], [(40, 300), (9, 130)]], ids=["one", "chunk"])
@pytest.mark.parametrize("P,D", [(16, 128), (32, 128), (64, 64)])
def test_missing_pages_beside_a_first_page_never_written(k_byte, v_byte, pairs, P, D):
    seq = _sequences(pairs, P, P)
    cache = r.random_cache(seq, 2, D, 3)
    cache[2][0], cache[3][0] = k_byte, v_byte
    seq.table[0, 2], seq.table[1, 0], seq.table[0, -1] = -1, 1 << 30, seq.table[0, -1]
    _check(seq, cache, torch.randn(seq.T, 4, D, generator=r.gen(4)).bfloat16())


@pytest.mark.parametrize("k_byte,v_byte", BYTES)
@pytest.mark.parametrize("pairs", [[(1, 300), (1, 130)], [(40, 300), (9, 130)]], ids=["one", "chunk"])
@pytest.mark.parametrize("P,D", [(16, 128), (32, 128), (16, 64)])
def test_pages_just_before_the_window(k_byte, v_byte, pairs, P, D):
    window = 70
    seq = _sequences(pairs, P, P)
    cache = r.random_cache(seq, 2, D, 3)
    reached = 0
    for b, (n, length) in enumerate(pairs):
        first = length - n - window + 1   # the first token that a row sees
        for w in range(first // P):
            page = int(seq.table[b, w])
            cache[0][page], cache[1][page], cache[2][page], cache[3][page] = 0x7F, 0xFF, k_byte, v_byte
            reached += w * P + P > first // 64 * 64   # (in the first tile of 64)
    assert reached > 0
    _check(seq, cache, torch.randn(seq.T, 4, D, generator=r.gen(4)).bfloat16(), window)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("pairs", [[(1, 200)], [(40, 200)]], ids=["one", "chunk"])
def test_rows_that_see_no_page_are_zero_whatever_their_queries(value, pairs):
    seq = _sequences(pairs, 16, 1)
    cache = r.random_cache(seq, 2, 128, 3)
    seq.table[:] = -1
    q = torch.randn(seq.T, 4, 128, generator=r.gen(4)).bfloat16()
    q[:, 0, 3] = value
    got = layer.attention(r.to_device(cache), seq.batch(), q.to(r.DEV))
    assert not bool(got.any())
