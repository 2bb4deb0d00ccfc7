"""gemm8 against 64 bits: odd sizes, ends of blocks, strides, scales, NaN beside the operands."""
import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


def _inputs(M, N, K, seed, pad=0):
    """Weights and rows inside wider arrays whose other columns hold NaN."""
    g = r.gen(seed)
    wide = K + 16 * pad
    w = torch.full((N, wide), 0x7F, dtype=torch.uint8)
    w[:, :K] = (torch.randn(N, K, generator=g) * 100).clamp(-448, 448).to(r.E4M3).view(torch.uint8)
    x = torch.full((M, wide), 0x7F, dtype=torch.uint8)
    x[:, :K] = (torch.randn(M, K, generator=g) * 100).clamp(-448, 448).to(r.E4M3).view(torch.uint8)
    nb, kb = -(-N // 128), -(-K // 128)
    ws = torch.rand(nb, kb, generator=g) * 1e-3 + 1e-5
    ws[0, 0] = -ws[0, 0]
    xs = torch.randint(110, 130, (M, kb), generator=g).to(torch.uint8)
    return w, ws, x, xs


def _product(w, ws, x, xs, K):
    """(product, what the instruction's sums may lose): it adds groups of eight products in units of 2^-13 of the largest of them, rounded down."""
    N = w.shape[0]
    wv = r.values(w[:, :K].contiguous()) * ws.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    xv = r.values(x[:, :K].contiguous()) * torch.exp2(xs.double() - 127).repeat_interleave(128, 1)[:, :K]
    lost = torch.zeros(x.shape[0], N, dtype=torch.float64)
    xg, wg = xv.abs().float().view(-1, K // 8, 8), wv.abs().float().view(N, K // 8, 8)
    for g in range(K // 8):
        lost += (xg[:, None, g] * wg[None, :, g]).amax(2).double()
    return xv @ wv.t(), lost * 7 * 2.0 ** -13


def _check(got, want, lost, K):
    # bf16 rounding is up to 2^-8 of the value; the fp32 sums of groups and blocks are below what the instruction loses within a group
    d = got.double().cpu() - want
    assert bool((d.abs() <= (2.0 ** -8 + 2.0 ** -18) * want.abs() + lost).all())
    # and over all outputs little more than bf16's rounding, 2^-8 / sqrt(3) of the value's binade: 0.0017 of normal numbers
    if want.numel() >= 4096 and bool(want.isfinite().all()):
        assert float(d.norm() / want.norm()) < 2.0 ** -9


SHAPES = [(1, 16, 16), (1, 1, 128), (1, 5001, 272), (2, 128, 2064), (5, 130, 384), (16, 257, 1040), (17, 500, 1024), (31, 96, 4112), (33, 1000, 640), (64, 333, 768), (65, 512, 512),
          (100, 129, 144), (128, 256, 2048), (129, 384, 1168), (200, 1100, 1552), (256, 256, 128), (257, 511, 400), (300, 2000, 976), (513, 770, 528), (777, 1025, 656), (1024, 640, 1152)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("pad", [0, 3])
def test_product(M, N, K, pad):
    w, ws, x, xs = _inputs(M, N, K, M + N + K, pad)
    want, lost = _product(w, ws, x, xs, K)
    weight = layer.Weight8(w.to(r.DEV)[:, :K], ws.to(r.DEV))
    rows = layer.Rows8(x.to(r.DEV)[:, :K], xs.to(r.DEV))
    out = torch.full((M, (N + 15) // 8 * 8), 7.0, dtype=torch.bfloat16, device=r.DEV)
    got = layer.gemm8(weight, rows, out=out[:, :N])
    _check(got, want, lost, K)
    assert bool((out[:, N:] == 7).all())
    assert torch.equal(layer.gemm8(weight, rows), got)   # its own output, the same every time


def test_rows_of_float8_types_and_bf16_rows():
    M, N, K = 40, 384, 896
    w, ws, _, _ = _inputs(M, N, K, 5)
    x = torch.randn(M, K, generator=r.gen(6)).bfloat16()
    weight = layer.Weight8(w.to(r.DEV).view(torch.float8_e4m3fn), ws.to(r.DEV))
    rows = layer.quantize8(x.to(r.DEV))
    got = layer.gemm8(weight, x.to(r.DEV))
    assert torch.equal(got, layer.gemm8(weight, rows))
    assert torch.equal(got, layer.gemm8(weight, layer.Rows8(rows.codes.view(torch.float8_e4m3fn), rows.scales.view(torch.float8_e8m0fnu))))
    want, lost = _product(w, ws, rows.codes.cpu(), rows.scales.cpu(), K)
    _check(got, want, lost, K)


@pytest.mark.parametrize("M", [1, 20, 70, 300])
def test_nan_rows_stay_in_their_row(M):
    N, K = 200, 400
    w, ws, x, xs = _inputs(M, N, K, 9)
    clean = layer.gemm8(layer.Weight8(w.to(r.DEV), ws.to(r.DEV)), layer.Rows8(x.to(r.DEV), xs.to(r.DEV))).cpu()
    x[M // 2, 256:] = 0x7F   # the last block, as the quantizer leaves a block with a NaN in it
    xs[M // 2, 2:] = 255
    xs[M // 2, 3] = 255
    got = layer.gemm8(layer.Weight8(w.to(r.DEV), ws.to(r.DEV)), layer.Rows8(x.to(r.DEV), xs.to(r.DEV))).cpu()
    assert bool(got[M // 2].isnan().all())
    others = torch.arange(M) != M // 2
    assert torch.equal(got[others], clean[others])


def test_no_rows_and_one_value_everywhere():
    w = layer.Weight8(torch.full((40, 160), 0x38, dtype=torch.uint8, device=r.DEV), torch.ones(1, 2, device=r.DEV))   # 0x38 is 1.0
    assert layer.gemm8(w, torch.empty(0, 160, dtype=torch.bfloat16, device=r.DEV)).shape == (0, 40)
    for M in (1, 33, 400):
        assert bool((layer.gemm8(w, torch.ones(M, 160, dtype=torch.bfloat16, device=r.DEV)) == 160).all())


def test_another_stream():
    w, ws, _, _ = _inputs(8, 512, 1024, 11)
    weight = layer.Weight8(w.to(r.DEV), ws.to(r.DEV))
    x = torch.randn(300, 1024, generator=r.gen(12)).bfloat16().to(r.DEV)
    want = layer.gemm8(weight, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = layer.gemm8(weight, x, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("M", [1, 7, 16, 40, 64, 90, 150, 400, 1100])
@pytest.mark.parametrize("N,K", [(300, 1040), (5001, 2000), (2048, 7168)])
def test_bf16_rows(M, N, K):
    """The bits of quantize8 and the product, through the native path, the general one with a stream, and a workspace of the caller's."""
    w, ws, _, _ = _inputs(1, N, K, 21)
    weight = layer.Weight8(w.to(r.DEV), ws.to(r.DEV))
    x = torch.randn(M, K + 3, generator=r.gen(22)).bfloat16().to(r.DEV)[:, 1:K + 1]
    got = layer.gemm8(weight, x)
    want, size = x.double() @ r.values(w).to(r.DEV).mul(ws.repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K].double().to(r.DEV)).t(), None
    # a value's rounding is 2^-4 of it at most, independent from value to value: the norm of the error is far below that of the result
    assert ((got.double() - want).norm() / want.norm()).item() < 2.0 ** -4
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = layer.gemm8(weight, x, stream=s)
    s.synchronize()
    need = layer.gemm8_workspace_bytes(weight, M, True)
    given = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=r.DEV)
    own = layer.gemm8(weight, x, workspace=given[:need] if need else None)
    assert torch.equal(other, got) and torch.equal(own, got) and bool((given[need:] == 0xFF).all())
