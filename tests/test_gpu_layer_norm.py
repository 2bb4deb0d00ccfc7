"""rms_norm and quantize8 against 64 bits: types, odd sizes and strides, every launch shape, in-place results, NaN and infinities."""
import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import binding as b
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _norm(h, w):
    return h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * w


def _check_y(got, want):
    # bf16 rounding is up to 2^-8 of the value; the fp32 steps before it (a sum of up to 40000 squares in a tree, a square root, a division, two products) stay under 2^-20
    got = got.double().cpu()
    assert got.shape == want.shape
    assert bool(((got - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs() + 1e-38).all())


def _check_rows8(got, want):
    """want: fp64 rows.  A block whose largest magnitude is within 2^-18 of the next scale may have either."""
    units, exps = r.rows8(want)
    have = got.scales.cpu().long() - 127
    code = r.values(got.codes.contiguous())
    step = torch.exp2((have - exps).double())
    assert bool((have - exps).abs().max() <= 1)
    for m, c in torch.nonzero(have != exps).tolist():
        top = float(want[m, c * 128:(c + 1) * 128].abs().max()) * 2.0 ** -float(min(have[m, c], exps[m, c]))
        assert abs(top / 448.0 - 1) < 2.0 ** -18
    units = units / step.repeat_interleave(128, 1)[:, :units.shape[1]]
    # half a step: 2^-4 of the value, or 2^-10 below e4m3's smallest normal number
    assert bool(((code - units).abs() <= units.abs() * (2.0 ** -4 + 2.0 ** -17) + 2.0 ** -10 * (1 + 2.0 ** -10)).all())


# every launch shape: 64, 256, 1024 threads a row with 1, 2, 4 pieces each, and rows of any length
SIZES = [(1, 1), (3, 7), (2, 64), (5, 129), (1, 512), (7, 520), (600, 513), (513, 1024), (520, 1999), (513, 2048), (2, 2056), (515, 2049), (513, 4104), (512, 8192), (1, 8192),
         (3, 8200), (2, 16384), (2, 16392), (1, 32768), (2, 33001), (1, 40000)]


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("residual", [None, torch.bfloat16, torch.float32])
def test_norm(M, N, residual):
    g = r.gen(M * 7 + N)
    x = torch.randn(M, N, generator=g).bfloat16()
    x[:, ::5] *= 8
    w = (1 + 0.2 * torch.randn(N, generator=g)).to(torch.bfloat16 if N % 2 else torch.float32)
    res = None if residual is None else (3 * torch.randn(M, N, generator=g)).to(residual)
    h = x.double() if res is None else x.double() + res.double()
    want = _norm(h, w.double())
    xd, wd = x.to(r.DEV), w.to(r.DEV)
    rd = None if res is None else res.to(r.DEV)
    sum_out = None if res is None else torch.full_like(rd, float("nan"))
    _check_y(layer.rms_norm(xd, wd, EPS, residual=rd, residual_out=sum_out), want)
    if res is not None:
        assert torch.equal(sum_out.cpu(), (x.float() + res.float()).to(residual))
        assert torch.equal(rd.cpu(), res)
    y = torch.empty_like(xd)
    got = layer.rms_norm(xd, wd, EPS, residual=rd, out=y, rows8=True)   # in place now, both results
    _check_y(y, want)
    _check_rows8(got, want)
    if res is not None:
        assert torch.equal(rd.cpu(), (x.float() + res.float()).to(residual))


@pytest.mark.parametrize("M,N", [(1, 1), (3, 17), (2, 128), (37, 7184), (513, 1030), (600, 300), (2, 40001)])
def test_quantize8_is_exact(M, N):
    g = r.gen(N)
    x = (torch.randn(M, N, generator=g) * torch.exp2(torch.randint(-20, 20, (M, N), generator=g).float() / 4)).bfloat16()
    x[0, : N // 2] = 0
    got = layer.quantize8(x.to(r.DEV))
    units, exps = r.rows8(x.double())
    zero = units.new_tensor([[bool((x[m, c * 128:(c + 1) * 128] == 0).all()) for c in range(exps.shape[1])] for m in range(M)]).bool()
    assert torch.equal(got.scales.cpu().long() - 127, torch.where(zero, torch.full_like(exps, -126), exps))
    assert torch.equal(r.values(got.codes.contiguous()), r.round_e4m3(units))


def test_quantize8_largest_and_smallest():
    """Blocks at the line between two scales, the largest bf16, subnormal numbers, zeros."""
    top = torch.tensor([448.0, 450.0, 446.0, 1.75, 1.7578125, 3.3895e38, 1e-40, 2.0 ** -126 * 448, 2.0 ** -127 * 448]).bfloat16()
    x = torch.zeros(top.numel(), 256).bfloat16()
    x[:, 3] = top
    x[:, 200] = -top
    got = layer.quantize8(x.to(r.DEV))
    units, exps = r.rows8(x.double())
    assert torch.equal(got.scales.cpu().long() - 127, exps)
    assert torch.equal(r.values(got.codes), r.round_e4m3(units))


def test_nan_and_infinities_stay_in_their_block_or_row():
    x = torch.randn(4, 300, generator=r.gen(1)).bfloat16()
    x[1, 130], x[2, 5] = float("nan"), float("inf")
    got = layer.quantize8(x.to(r.DEV))
    s, c = got.scales.cpu(), r.values(got.codes.contiguous())
    bad = torch.zeros(4, 3, dtype=torch.bool)
    bad[1, 1] = bad[2, 0] = True
    assert torch.equal(s == 255, bad)
    assert torch.equal(c.isnan(), bad.repeat_interleave(128, 1)[:, :300])
    y = layer.rms_norm(x.to(r.DEV), None, EPS).cpu()
    assert bool(y[1].isnan().all()) and bool(y[2, 5].isnan()) and bool((y[2, :5] == 0).all()) and bool(y[[0, 3]].isfinite().all())
    n = layer.rms_norm(x.to(r.DEV), None, EPS, rows8=True)
    assert bool((n.scales[1].cpu() == 255).all()) and n.scales[2].cpu().tolist()[0] == 255 and 255 not in n.scales[0].tolist()


def test_strides_rows_and_columns_beside_are_left_alone():
    """Rows of a wider tensor at an odd column, results into one, nothing beside them written."""
    M, N = 9, 203
    big = torch.randn(M, 3 * N + 1, generator=r.gen(3)).bfloat16().to(r.DEV)
    x, res = big[:, 1:1 + N], big[:, N + 1:2 * N + 1]
    out = torch.full((M, N + 5), 7.0, dtype=torch.bfloat16, device=r.DEV)
    total = torch.full((M, N + 3), 7.0, dtype=torch.bfloat16, device=r.DEV)
    h = (x.float() + res.float()).double().cpu()
    got = layer.rms_norm(x, None, EPS, residual=res, residual_out=total[:, 1:N + 1], out=out[:, 2:N + 2])
    _check_y(got, _norm(h, 1.0))
    assert bool((out[:, :2] == 7).all()) and bool((out[:, N + 2:] == 7).all())
    assert bool((total[:, 0] == 7).all()) and bool((total[:, N + 1:] == 7).all())
    y = x.clone()
    assert layer.rms_norm(y, None, EPS, out=y) is y   # in place
    _check_y(y, _norm(x.double().cpu(), 1.0))
    q = layer.Rows8(torch.full((M, 224), 9, dtype=torch.uint8, device=r.DEV), torch.full((M, 3), 9, dtype=torch.uint8, device=r.DEV))
    import ctypes
    d = layer.ccq_rows8(q.codes.data_ptr(), 224, q.scales.data_ptr(), 3)
    assert layer._load().ccq_quantize8(b._t_ptr(x), x.stride(0), M, N, ctypes.byref(d), b._stream_ptr(None)) == 0
    assert bool((q.codes[:, N:] == 9).all()) and bool((q.scales[:, 2] == 9).all())


def test_no_rows_and_another_stream():
    x = torch.empty(0, 128, dtype=torch.bfloat16, device=r.DEV)
    assert layer.rms_norm(x, None).shape == (0, 128) and layer.quantize8(x).shape == (0, 128)
    x = torch.randn(64, 4096, generator=r.gen(4)).bfloat16().to(r.DEV)
    want = layer.rms_norm(x, None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = layer.rms_norm(x, None, stream=s)
    with torch.cuda.stream(s):
        again = layer.rms_norm(x, None)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(again, want)
