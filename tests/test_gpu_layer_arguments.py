"""Arguments of the layer operators on the GPU: what the native path and the general one make of them is the same."""
import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


def test_scales_whose_rows_share_memory_are_refused():
    w = layer.Weight8(torch.zeros(64, 256, dtype=torch.uint8, device=r.DEV), torch.ones(1, 2, device=r.DEV))
    codes, one = torch.zeros(4, 256, dtype=torch.uint8, device=r.DEV), torch.full((1, 2), 127, dtype=torch.uint8, device=r.DEV)
    for kw in ({}, dict(stream=torch.cuda.current_stream())):
        with pytest.raises((ValueError, layer.CcqError)):
            layer.gemm8(w, layer.Rows8(codes, one.expand(4, 2)), **kw)
    assert layer.gemm8(w, layer.Rows8(codes, one.repeat(4, 1))).shape == (4, 64)


@pytest.mark.parametrize("general", [False, True])
def test_workspaces_on_the_host_or_in_pieces_are_refused(general):
    """Where a workspace would be written to: the refusal comes before any launch."""
    from paper_2507_07145_amd import binding as b
    from paper_2507_07145_amd import synth
    kw = dict(stream=torch.cuda.current_stream()) if general else {}
    bad = [torch.empty(8 << 20, dtype=torch.uint8), torch.empty(2, 8 << 20, dtype=torch.uint8, device=r.DEV)[:, ::2], torch.empty(8 << 20, 2, dtype=torch.uint8, device=r.DEV)[:, 0]]
    w = layer.Weight8(torch.zeros(512, 7168, dtype=torch.uint8, device=r.DEV), torch.ones(4, 56, device=r.DEV))
    x = torch.zeros(300, 7168, dtype=torch.bfloat16, device=r.DEV)
    assert layer.gemm8_workspace_bytes(w, 300, True) > 0
    seq = r.Sequences([(1, 5000)], 64)
    cache, batch, q = r.to_device(r.random_cache(seq, 1, 64, 1)), seq.batch(), torch.zeros(1, 4, 64, dtype=torch.bfloat16, device=r.DEV)
    two = b.quantize(torch.from_numpy(synth.weights_normal(512, 1024, synth.rng(0, 0))).to(r.DEV), b.NARROW)
    rows, offsets = torch.arange(300, dtype=torch.int32, device=r.DEV), torch.tensor([0, 300], dtype=torch.int32, device=r.DEV)
    for ws in bad:
        for call in (lambda: layer.gemm8(w, x, workspace=ws, **kw), lambda: layer.attention(cache, batch, q, workspace=ws, **kw),
                     lambda: b.gemm(two, x[:, :1024], workspace=ws, **kw), lambda: b.grouped_gemm(two, x[:, :1024], rows, offsets, workspace=ws, **kw)):
            with pytest.raises(ValueError, match="workspace"):
                call()


def _memory_of(t):
    """The stream whose memory pool a tensor lies in."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("no segment holds the tensor")


def test_results_on_another_stream_come_from_its_memory():
    """The current stream's memory may still be read there, by kernels under way whose tensors were dropped; another stream must not write it."""
    s = torch.cuda.Stream()
    x = torch.randn(20, 256, generator=r.gen(0)).bfloat16().to(r.DEV)
    w = layer.Weight8(torch.zeros(64, 256, dtype=torch.uint8, device=r.DEV), torch.ones(1, 2, device=r.DEV))
    seq = r.Sequences([(3, 90)], 16)
    cache, batch = r.to_device(r.random_cache(seq, 1, 64, 1)), seq.batch()
    q = torch.randn(3, 4, 64, generator=r.gen(1)).bfloat16().to(r.DEV)
    s.wait_stream(torch.cuda.current_stream())
    rows, q8 = layer.rms_norm(x, None, rows8=True, stream=s), layer.quantize8(x, stream=s)
    made = [layer.rms_norm(x, None, stream=s), rows.codes, rows.scales, q8.codes, q8.scales, layer.gemm8(w, x, stream=s), layer.gemm8(w, q8, stream=s),
            layer.attention(cache, batch, q, stream=s), layer.cache_append(cache, batch, None, None, q=q, stream=s), layer.rope_table(10, 8, stream=s)]
    s.synchronize()
    assert [_memory_of(t) for t in made] == [s.cuda_stream] * len(made)
    assert _memory_of(layer.rms_norm(x, None)) == torch.cuda.current_stream().cuda_stream
    assert torch.equal(made[1], layer.rms_norm(x, None, rows8=True).codes) and torch.equal(made[8], q) and torch.equal(made[9], layer.rope_table(10, 8))


@pytest.mark.parametrize("true,false", [(1, 0), (torch.tensor(True), torch.tensor(False))], ids=["int", "tensor"])
def test_flags_by_their_truth(true, false):
    """What is true is true on the native path and the general one, be it True itself or not."""
    seq = r.Sequences([(5, 90), (1, 40)], 16)
    cache, batch = r.to_device(r.random_cache(seq, 1, 64, 1)), seq.batch()
    q = torch.randn(6, 4, 64, generator=r.gen(7)).bfloat16().to(r.DEV)
    causal, whole = layer.attention(cache, batch, q, causal=True), layer.attention(cache, batch, q, causal=False)
    assert not torch.equal(causal, whole)
    x = torch.randn(2, 256, generator=r.gen(2)).bfloat16().to(r.DEV)
    for kw in ({}, dict(stream=torch.cuda.current_stream())):
        assert torch.equal(layer.attention(cache, batch, q, causal=true, **kw), causal)
        assert torch.equal(layer.attention(cache, batch, q, causal=false, **kw), whole)
        assert torch.equal(layer.rms_norm(x, None, rows8=true, **kw).codes, layer.rms_norm(x, None, rows8=True).codes)
        assert torch.equal(layer.rms_norm(x, None, rows8=false, **kw), layer.rms_norm(x, None))


def test_rows_of_four_million_values():
    """A product whose row scales pass the LDS if the streaming kernel takes it: ones times ones, exact in every order of sums."""
    K, N = 1 << 22, 2048
    w = layer.Weight8(torch.full((N, K), 0x38, dtype=torch.uint8, device=r.DEV), torch.ones(N // 128, K // 128, device=r.DEV))   # 0x38 is 1.0
    for M in (16, 64):
        rows = layer.Rows8(torch.full((M, K), 0x38, dtype=torch.uint8, device=r.DEV), torch.full((M, K // 128), 127, dtype=torch.uint8, device=r.DEV))
        assert bool((layer.gemm8(w, rows) == K).all())
        assert bool((layer.gemm8(w, torch.ones(M, K, dtype=torch.bfloat16, device=r.DEV)) == K).all())


def test_windows_past_32_bits_are_refused():
    """Cut off to 32 bits, 2^32 + 5 would be a window of 5."""
    seq = r.Sequences([(1, 40)], 16)
    cache, batch, q = r.to_device(r.random_cache(seq, 1, 64, 1)), seq.batch(), torch.zeros(1, 4, 64, dtype=torch.bfloat16, device=r.DEV)
    for kw in ({}, dict(stream=torch.cuda.current_stream())):
        with pytest.raises(ValueError, match="31 bits"):
            layer.attention(cache, batch, q, window=(1 << 32) + 5, **kw)
        assert layer.attention(cache, batch, q, window=(1 << 31) - 1, **kw).shape == q.shape
