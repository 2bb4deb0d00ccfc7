"""The rule of the 8-bit product offers only what can be launched.  Host only."""
import ctypes

import pytest

from paper_2507_07145_amd import layer

STREAM = 1


def plan(M, N, K):
    out, time = (ctypes.c_int32 * 7)(), ctypes.c_double()
    layer._load().ccq_gemm8_plan(M, N, K, out, ctypes.byref(time))
    return list(out)


@pytest.mark.parametrize("K", [1 << 17, 200000, 1 << 18, 400000, 1 << 20, 1 << 21, 1 << 22, (1 << 23) + 16, 1 << 26])
def test_scales_of_a_share_fit_the_lds(K):
    """The streaming kernel holds its share's row scales in LDS beside two steps of activations: 160 KB in all."""
    streams = 0
    for N in (16, 128, 512, 2048, 8192, 16384, 32768, 65536, 131072):
        for M in (1, 4, 16, 17, 24, 32, 33, 48, 64, 65, 80, 96, 128, 160, 192):
            kind, mt, shares = plan(M, N, K)[:3]
            if kind == STREAM:
                streams += 1
                blocks = -(-K // 128)
                per_share = (-(-blocks // shares) + 1) // 2 * 2
                assert 2 * 16 * mt * 256 + 16 * mt * ((per_share + 7) // 4 * 4) <= 160 * 1024, (M, N, K, mt, shares)
    assert streams > 0 or K > 1 << 20


def test_a_named_plan_is_checked():
    """Calls as a plan of the test's choice: no such kernel, or arguments that the entry points refuse, and nothing is launched."""
    p = 4096   # a pointer that no call below may look behind
    f = layer._load().ccq_gemm8_as
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]

    def call(plan, M=40, w={}, x={}, y=p, ldy=600, ws=p):
        wd = layer.ccq_weight8(**{**dict(K=256, N=600, codes=p, ldw=256, scales=p, ld_scales=2), **w})
        xd = layer.ccq_rows8(**{**dict(codes=p, ld=256, scales=p, ld_scales=2), **x})
        return f(ctypes.byref(wd), ctypes.byref(xd), M, y, ldy, ws, (ctypes.c_int32 * 7)(*plan), None)

    bad, null, align, workspace = -2, -1, -4, -5
    for plan in ([0, 2, 1, 4, 0, 0, 1], [0, 1, 1, 8, 0, 0, 1], [0, 4, 1, 16, 0, 0, 1], [0, 4, 2, 4, 0, 0, 1], [1, 5, 1, 4, 0, 0, 1], [1, 2, 0, 4, 0, 0, 1], [2, 3, 1, 4, 0, 0, 1],
                 [2, 4, 0, 4, 0, 0, 1], [2, 4, 1, 4, 100, 1, 1], [2, 4, 1, 4, 768, 1, 1], [2, 4, 2, 4, 256, 1, 1], [2, 4, 1, 4, 256, 3, 1], [1, 2, 1, 4, 256, 1, 1], [3, 1, 1, 4, 0, 0, 1]):
        assert call(plan) == bad, plan
    few = [0, 4, 1, 4, 0, 0, 1]
    assert call(few, y=None) == null and call(few, y=p + 8) == align and call(few, ldy=592) == bad and call(few, w=dict(codes=None)) == null and call(few, M=-1) == bad
    assert call(few, x=dict(ld=128)) == bad and call(few, x=dict(scales=None, ld=255)) == bad and call(few, x=dict(scales=None, codes=p + 1)) == align
    assert call([2, 1, 2, 4, 0, 0, 1], ws=None) == workspace and call([1, 6, 1, 4, 0, 0, 1], x=dict(scales=None)) == bad and call([2, 1, 1, 4, 0, 0, 1], x=dict(scales=None)) == bad
    assert call([2, 1, 1, 4, 0, 0, 1], w=dict(ldw=1 << 24)) == bad and call(few, M=0) == 0
