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
