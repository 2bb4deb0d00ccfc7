"""Adapters up to 511 rows, and of few results: workgroups of the MFMA kernel that go over several pieces of columns, in each of its four widths of ranks, on both sides of
where a CU has room for one of them instead of two (ranks of 216 and 224)."""
import pytest
import torch

from paper_2507_07145_amd import routing
from test_gpu_adapters import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# rows, columns, rank, adapters, runs (0: rows of every adapter mixed); pieces of 256 columns (128 above rank 64) of a workgroup
CASES = [
    (300, 8201, 24, 4, 0),      # 2 of 33
    (500, 5000, 24, 100, 0),    # 7 of 20
    (511, 8201, 64, 4, 5),      # 3 of 33
    (480, 3001, 64, 90, 0),     # 3 of 12
    (3000, 1000, 64, 40, 70),   # 2 of 4
    (260, 8201, 96, 4, 4),      # 3 of 65
    (256, 8200, 136, 4, 0),     # 3 of 65
    (300, 4100, 216, 5, 6),     # 2 of 33
    (300, 4100, 224, 5, 6),     # 4 of 33
    (400, 8201, 256, 3, 3),     # 8 of 65
    (40, 8193, 256, 4, 0),      # 2 of 65
]


@pytest.mark.parametrize("T,N,R,n,runs", CASES)
@pytest.mark.parametrize("ranks", [False, True])
def test_several_pieces(T, N, R, n, runs, ranks):
    c = Case(T, 136, N, R, n, T + N + R, ranks=ranks, runs=runs)
    adapters, order, x, y = c.set(), c.order(), c.x.to(DEV), c.y.to(DEV)
    got = routing.adapters(y, x, adapters, order)
    c.check(got, f"{T} rows to {N}, {n} adapters of {R}")
    wide = torch.full((T, N + 9), 3.0, dtype=torch.bfloat16, device=DEV)      # in place, in columns of wider rows
    wide[:, 5:5 + N] = y
    routing.adapters(wide[:, 5:5 + N], x, adapters, order, out=wide[:, 5:5 + N])
    assert torch.equal(wide[:, 5:5 + N], got)
    assert bool((wide[:, :5] == 3.0).all()) and bool((wide[:, 5 + N:] == 3.0).all())
