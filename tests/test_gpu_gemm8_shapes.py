"""Every launch shape of gemm8 against 64 bits, whatever the rule would choose, and the rule's choices where two of them meet."""
import ctypes

import pytest
import torch

import layer_ref as r
import test_gpu_gemm8 as t
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu
FEW, STREAM, BLOCK = 0, 1, 2


def _as(weight, rows, M, N, plan):
    f = layer._load().ccq_gemm8_as
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    y = torch.full((M, (N + 15) // 8 * 8), 7.0, dtype=torch.bfloat16, device=r.DEV)
    ws = torch.full((max(plan[2], plan[6]) * M * ((N + 3) // 4 * 4) * 4 + 64,), 0xFF, dtype=torch.uint8, device=r.DEV)   # NaN
    d = rows.desc()
    rc = f(ctypes.byref(weight.desc), ctypes.byref(d), M, y.data_ptr(), y.stride(0), ws.data_ptr(), (ctypes.c_int32 * 7)(*plan), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert bool((y[:, N:] == 7).all()) and bool((ws[-64:] == 0xFF).all())
    return y[:, :N]


def _as_bf16(weight, x, N, plan):
    """The same with bf16 rows."""
    class Rows:
        @staticmethod
        def desc():
            return layer.ccq_rows8(x.data_ptr(), x.stride(0), None, 0)
    return _as(weight, Rows, x.shape[0], N, plan)


def plan(M, N, K):
    out, time = (ctypes.c_int32 * 7)(), ctypes.c_double()
    layer._load().ccq_gemm8_plan(M, N, K, out, ctypes.byref(time))
    return list(out)


PLANS = ([[FEW, 1, 1, 4, 0, 0, 1], [FEW, 1, 1, 16, 0, 0, 1], [FEW, 4, 1, 4, 0, 0, 1]] + [[STREAM, mt, s, 4, 0, 0, 1] for mt in (1, 2, 3, 4, 6) for s in (1, 2, 5)] +
         [[BLOCK, mi, s, 4, 0, 0, 1] for mi in (1, 2, 4) for s in (1, 3)] + [[BLOCK, 4, 1, 4, 256, 1, 1], [BLOCK, 4, 1, 4, 256, 2, 3], [BLOCK, 2, 1, 4, 512, 4, 2]])


@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (5, 130, 384), (37, 601, 1936), (64, 333, 768), (100, 129, 144), (129, 1100, 1552), (257, 513, 1040)])
@pytest.mark.parametrize("p", PLANS, ids=str)
def test_shape(M, N, K, p):
    if p[4] >= N:
        pytest.skip("no columns are left for the second part")
    w, ws, x, xs = t._inputs(M, N, K, M + N + K, 3)
    want, lost = t._product(w, ws, x, xs, K)
    got = _as(layer.Weight8(w.to(r.DEV)[:, :K], ws.to(r.DEV)), layer.Rows8(x.to(r.DEV)[:, :K], xs.to(r.DEV)), M, N, p)
    t._check(got, want, lost, K)


@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (5, 130, 384), (37, 601, 1936), (64, 333, 768), (100, 129, 144), (129, 300, 1552)])
@pytest.mark.parametrize("p", [q for q in PLANS if q[0] == FEW or (q[0] == STREAM and q[1] <= 4)], ids=str)
def test_bf16_rows_give_the_bits_of_their_8_bit_rows(M, N, K, p):
    w, ws, _, _ = t._inputs(M, N, K, M + N + K, 3)
    wide = torch.randn(M, K + 5, generator=r.gen(M)).mul(torch.randn(M, 1, generator=r.gen(N)).mul(8).exp2()).bfloat16()
    wide[:, 3:3 + min(K, 100)] *= 2.0 ** -30
    if M > 2:
        wide[1, K // 2] = float("nan")
        wide[2, 3] = float("-inf")
        wide[M - 1] = 0
    x = wide.to(r.DEV)[:, 3:3 + K]   # (rows that start at odd addresses)
    weight = layer.Weight8(w.to(r.DEV)[:, :K], ws.to(r.DEV))
    want = _as(weight, layer.quantize8(x), M, N, p)
    assert torch.equal(_as_bf16(weight, x, N, p).contiguous().view(torch.int16), want.contiguous().view(torch.int16))


@pytest.mark.parametrize("p", [[BLOCK, 1, 1, 4, 0, 0, 1], [BLOCK, 2, 1, 4, 0, 0, 1], [BLOCK, 4, 1, 4, 0, 0, 1], [STREAM, 4, 1, 4, 0, 0, 1], [FEW, 1, 1, 16, 0, 0, 1]], ids=str)
def test_long_k(p):
    """More steps than the scales of 64 that lie in LDS at a time, and a ragged last one."""
    M, N, K = 70, 300, 128 * 131 + 48
    w, ws, x, xs = t._inputs(M, N, K, 1)
    want, lost = t._product(w, ws, x, xs, K)
    t._check(_as(layer.Weight8(w.to(r.DEV), ws.to(r.DEV)), layer.Rows8(x.to(r.DEV), xs.to(r.DEV)), M, N, p), want, lost, K)


def test_the_rule_reaches_every_kind():
    kinds = {tuple(plan(M, N, K)[:2]) for M in (1, 8, 16, 17, 33, 48, 64, 96, 128, 300, 1024, 2048) for N, K in ((8192, 8192), (28672, 8192), (5001, 7184), (18432, 7168), (1000, 1024))}
    assert {(FEW, 1), (FEW, 4), (STREAM, 1), (STREAM, 2), (STREAM, 3), (STREAM, 4), (STREAM, 6), (BLOCK, 1), (BLOCK, 2), (BLOCK, 4)} <= kinds
    assert plan(2048, 18432, 7168)[4] > 0   # two parts


def test_rows_far_apart():
    """Rows that 32-bit offsets within a block would not reach: a stride of 9 MiB."""
    M, N, K = 200, 40, 160
    w, ws, x, xs = t._inputs(M, N, K, 3)
    big = torch.zeros(M, (9 << 20), dtype=torch.uint8, device=r.DEV)
    big[:, :K] = x.to(r.DEV)
    want, lost = t._product(w, ws, x, xs, K)
    got = layer.gemm8(layer.Weight8(w.to(r.DEV), ws.to(r.DEV)), layer.Rows8(big[:, :K], xs.to(r.DEV)))
    t._check(got, want, lost, K)
