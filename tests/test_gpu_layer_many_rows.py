"""Calls of more workgroups than one launch may have (2^32 threads)."""
import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


def test_norm_of_more_rows_than_a_launch_has():
    """Heads of 16 values, four rows to a workgroup: 70 million of them."""
    M, N = 70_000_001, 16
    x = torch.randn(1 << 16, N, generator=r.gen(0)).bfloat16().to(r.DEV).repeat(M // (1 << 16) + 1, 1)[:M]
    w = torch.rand(N, generator=r.gen(1)).to(r.DEV)
    want, want8 = layer.rms_norm(x[:1 << 16], w), layer.rms_norm(x[:1 << 16], w, rows8=True)
    y = layer.rms_norm(x, w)
    y8 = layer.rms_norm(x, w, rows8=True)
    for first in range(0, M, 1 << 16):
        n = min(1 << 16, M - first)
        assert torch.equal(y[first:first + n], want[:n]) and torch.equal(y8.codes[first:first + n], want8.codes[:n]) and torch.equal(y8.scales[first:first + n], want8.scales[:n])
    h = x.clone()
    total = torch.full_like(x, 0.5)
    layer.rms_norm(h, w, residual=total, out=h)   # in place: sum and result
    one = torch.full_like(want, 0.5)
    first = layer.rms_norm(x[:1 << 16], w, residual=one)
    n = M % (1 << 16)
    assert torch.equal(total[-n:], one[:n]) and torch.equal(h[-n:], first[:n]) and torch.equal(total[:1 << 16], one) and torch.equal(h[:1 << 16], first)


def test_append_with_a_bound_on_new_tokens_of_many_workgroups():
    """520 sequences of one or three new tokens, of which a call may have 32768: 17 million workgroups, nearly all of them empty."""
    pairs = [(1, 5 + i % 40) for i in range(519)] + [(3, 30)]
    seq = r.Sequences(pairs, 16)
    k, v = (torch.randn(seq.T, 1, 64, generator=r.gen(i)).bfloat16().to(r.DEV) for i in (1, 2))
    q = torch.randn(seq.T, 2, 64, generator=r.gen(3)).bfloat16().to(r.DEV)
    rope = layer.Rope(layer.rope_table(64, 64))
    empty = [torch.zeros_like(t) for t in r.random_cache(seq, 1, 64, 1)]
    near, far = r.to_device(empty), r.to_device(empty)
    b = seq.batch()
    want = layer.cache_append(near, b, k, v, q, rope=rope)
    wide = layer.Batch(b.offsets, b.lens, b.table, seq.T, 32768, seq.max_len)
    got = layer.cache_append(far, wide, k, v, q, rope=rope)
    assert torch.equal(got, want)
    for one, other in ((near.k, far.k), (near.v, far.v), (near.k_scales, far.k_scales), (near.v_scales, far.v_scales)):
        assert torch.equal(one, other)


def test_many_rows_on_weights_far_apart():
    """Weights whose rows are 9 MiB apart go to the kernel for few rows, whatever the rows' number: more of them than its grid has."""
    M, N, K = 65535 * 64 + 77, 16, 48
    big = torch.zeros(N, 9 << 20, dtype=torch.uint8, device=r.DEV)
    big[:, :K] = torch.randint(0, 0x60, (N, K), generator=r.gen(0), dtype=torch.uint8).to(r.DEV)
    far, near = layer.Weight8(big[:, :K], torch.ones(1, 1, device=r.DEV)), layer.Weight8(big[:, :K].contiguous(), torch.ones(1, 1, device=r.DEV))
    x = torch.randn(1 << 12, K, generator=r.gen(1)).bfloat16().to(r.DEV).repeat(M // (1 << 12) + 1, 1)[:M]
    want = layer.gemm8(near, x[:1 << 12])
    for rows in (x, layer.quantize8(x)):
        y = layer.gemm8(far, rows)
        for first in (0, 1 << 20, (65535 * 64 >> 12) << 12):
            n = min(1 << 12, M - first)
            assert torch.equal(y[first:first + n], want[:n])
