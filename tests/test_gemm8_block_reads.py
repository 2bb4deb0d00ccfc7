"""What the 8-bit block kernel reads of rows that end inside an eighth and of columns that end inside a block: never a byte past the last row, and
zeros in place of no column that there is.  Host only: the index arithmetic that the kernel shares."""
import ctypes

import pytest

from paper_2507_07145_amd import layer


def _source():
    f = layer._load().ccq_gemm8_block_source
    f.restype, f.argtypes = ctypes.c_int64, [ctypes.c_int32] * 3 + [ctypes.c_int64] + [ctypes.c_int32] * 2
    return f


@pytest.mark.parametrize("K", [16, 112, 128, 144, 176, 208, 240, 528, 656, 7184])
@pytest.mark.parametrize("rows", [1, 7, 8, 9, 16, 17, 63, 64, 100, 129, 183, 250, 256])
def test_reads_lie_inside_the_array(rows, K):
    source, k = _source(), (K - 1) // 128 * 128   # the last block of K
    for ld in (K, K + 48):
        for eighth in range(32):
            for lane in range(64):
                at = source(lane, eighth, rows - 1, ld, k, K)
                if at < 0:
                    continue
                row, column = divmod(at, ld)
                assert 0 <= row < rows and k <= column <= K - 16, (eighth, lane, row, column)
                if 8 * eighth + lane // 8 < rows:   # a row that there is: its own
                    assert row == 8 * eighth + lane // 8


@pytest.mark.parametrize("K", [144, 176, 528, 7184])
@pytest.mark.parametrize("rows", [1, 8, 21, 64, 250, 256])
def test_every_chunk_of_every_row_is_copied(rows, K):
    source, k = _source(), (K - 1) // 128 * 128
    for eighth in range((rows + 7) // 8):
        for sub in range(min(8, rows - 8 * eighth)):
            got = sorted(source(8 * sub + place, eighth, rows - 1, K, k, K) for place in range(8))
            there = (K - k) // 16
            assert got == [-1] * (8 - there) + [(8 * eighth + sub) * K + k + 16 * c for c in range(there)]
