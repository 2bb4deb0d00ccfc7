"""Every kernel of the attention on every kind of call, whatever the rule would choose."""
import pytest
import torch

import layer_ref as r
import test_gpu_attention8 as t
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1], ids=["few", "many"])
def kernel(request):
    layer._load().ccq_attention_force(request.param)
    yield
    layer._load().ccq_attention_force(-1)


@pytest.mark.parametrize("pairs,P,D,Hkv,Hq,window,causal", [
    ([(1, 1)], 16, 64, 1, 1, 0, True), ([(1, 200), (1, 3), (1, 0), (1, 130)], 32, 128, 2, 14, 0, True), ([(1, 3000)], 64, 128, 1, 8, 0, True),
    ([(3, 70), (5, 5), (1, 40), (0, 9)], 16, 128, 2, 6, 0, True), ([(33, 33), (17, 100)], 32, 64, 2, 2, 20, True), ([(70, 70)], 64, 128, 1, 7, 0, True),
    ([(130, 400), (9, 900)], 64, 128, 1, 4, 100, True), ([(200, 333)], 128, 64, 2, 4, 0, False), ([(270, 300)], 16, 128, 1, 1, 0, True), ([(60, 700)], 256, 64, 1, 5, 64, True),
])
def test_call(kernel, pairs, P, D, Hkv, Hq, window, causal):
    t._run(pairs, P, D, Hkv, Hq, window, causal, seed=P + Hq)


@pytest.mark.parametrize("pairs", [[(1, 600)], [(40, 300)]])
def test_scales_far_apart_and_peaks(kernel, pairs):
    t.test_scales_far_apart(pairs, 3)
    t.test_peaked_rows(pairs, 2)


def test_pages_that_are_not_there(kernel):
    t.test_pages_that_are_not_there([(20, 200), (8, 90)])


def test_nan(kernel):
    t.test_nan_in_queries_and_keys_reach_the_rows_that_see_them()


def test_bounds(kernel):
    t.test_lengths_past_the_bounds_and_the_table()


def test_more_rows_than_a_tile_in_splits(kernel):
    """Few sequences and long: the cached tokens are cut, rows of several tiles."""
    t._run([(45, 5000)], 64, 128, 1, 2, seed=3)


def test_offsets_past_32_bits(kernel):
    t.test_offsets_past_32_bits()


def test_strides_and_another_stream(kernel):
    t.test_strides_and_the_general_path()


def test_a_captured_call(kernel):
    """Replays give the eager bits, with lengths and queries that change between them."""
    pairs, P, D, Hkv, Hq = [(40, 700), (3, 90)], 64, 128, 2, 8
    seq = r.Sequences(pairs, P, 11)
    cache = r.to_device(r.random_cache(seq, Hkv, D, 12))
    batch = seq.batch()
    q = torch.randn(seq.T, Hq, D, generator=r.gen(13)).bfloat16().to(r.DEV)
    first, second = q.clone(), q.flip(0).contiguous()
    lens = batch.lens.clone()
    eager = [layer.attention(cache, batch, first).clone(), layer.attention(cache, batch, second).clone()]
    batch.lens.copy_(lens - 33)
    eager.append(layer.attention(cache, batch, second).clone())
    batch.lens.copy_(lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.attention(cache, batch, q)
    for i in (0, 1, 2, 1, 0):
        q.copy_(first if i == 0 else second)
        batch.lens.copy_(lens - 33 if i == 2 else lens)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager[i].view(torch.int16))
        torch.randn(1 << 16, device=r.DEV).sum().item()


def _workspace(n, length, Hkv, Hq, D=128, window=0, B=1):
    import ctypes
    cache = layer.ccq_cache(64, 64, Hkv, D, None, None, None, None)
    batch = layer.ccq_batch(B, B * n, n, length, None, None, None, 1 << 20, 1 << 20)
    return layer._load().ccq_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(layer.ccq_attn(Hq, 1, window, 1.0)))


def test_the_rule_reaches_every_kernel():
    image = 4 * 64 * 128   # bytes of 64 tokens of a head
    assert _workspace(2048, 4096, 8, 56) >= 64 * 8 * image      # many rows
    assert _workspace(2048, 4096, 8, 56, D=64) == 0             # heads of 64: the kernel for few, enough of them
    assert _workspace(1, 200, 8, 32) == 0                       # one launch
    assert 0 < _workspace(1, 131072, 8, 64) < 64 << 20          # pieces of a long sequence
    assert _workspace(2048, 1 << 20, 8, 32, B=16) < 4 << 30     # images of all these tokens would be 16 times that


def test_a_chunk_as_the_rule_serves_it():
    t._run([(700, 1100)], 64, 128, 4, 32, seed=21)
    t._run([(500, 900), (130, 640)], 32, 128, 8, 32, window=300, seed=22)


@pytest.mark.parametrize("pairs", [[(1, 900)], [(1, 2500), (1, 30), (1, 0), (1, 1300)], [(40, 700), (3, 2000)]])
def test_a_bound_far_above_the_lengths(pairs):
    """max_len is what a table could hold: the pieces go by the lengths."""
    seq = r.Sequences(pairs, 64, 31)
    cache = r.random_cache(seq, 2, 128, 32)
    q = torch.randn(seq.T, 8, 128, generator=r.gen(33)).bfloat16()
    batch = seq.batch()
    far = layer.Batch(batch.offsets, batch.lens, batch.table, seq.T, max(n for n, _ in pairs), 1 << 17)
    got = layer.attention(r.to_device(cache), far, q.to(r.DEV)).cpu().double()
    want, size = r.attend(seq, cache, q, 128 ** -0.5)
    assert bool(((got - want).abs() <= r.attend_limit(want, size)).all())
