"""A router's choice where scores are equal in 64 bits and logits are not."""
import pytest
import torch

from test_gpu_route import check, logits_of

pytestmark = pytest.mark.gpu


def rows_of(scoring):
    """Rows of 16 logits, four groups of four, whose groups' largest scores are equal in 64 bits although their logits are not."""
    inf, low = float("inf"), -float("inf")
    fill = lambda *best: [v for b in best for v in (b, b - 3.0 if abs(b) < inf else b, low, b)]  # noqa: E731
    rows = [fill(2.0 ** -70, 2.0 ** -60, 2.0 ** -80, 1.0), fill(-2.0 ** -70, 2.0 ** -90, 0.0, -1.0), fill(low, 2.0 ** -75, 2.0 ** -65, low)]
    if scoring == "sigmoid":   # 1 + e^-40 is 1, e^800 infinity
        rows += [fill(40.0, 50.0, 45.0, 60.0), fill(39.5, 1.0, 77.0, 41.0), fill(-800.0, -760.0, -790.0, -1000.0), fill(low, -800.0, -760.0, 0.5), fill(50.0, inf, 3e38, 60.0),
                 fill(-3e38, -1e30, -900.0, low), fill(20.0, 19.0, 18.0, 21.0)]
    else:                      # e^-760 is 0
        rows += [fill(0.0, -800.0, -760.0, -790.0), fill(-900.0, -800.0, 5.0, -760.0), fill(1e30, 3e38, 2e30, 0.0), fill(1.0, 2.0, inf, 3.0), fill(-1e30, -3e38, -2e30, low),
                 fill(-700.0, -720.0, 0.0, -710.0)]
    return torch.tensor(rows)


@pytest.mark.parametrize("scoring", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_groups_of_equal_scores_go_by_the_lower_index(scoring, dtype):
    rows = rows_of(scoring).to(dtype)
    for T in (len(rows), 100, 2100):      # eight rows and fewer, a wavefront for each row, 16 lanes
        l = logits_of(T, 16, T, dtype)
        at = torch.arange(0, T, max(1, T // len(rows)))[:len(rows)]
        l[at] = rows
        for best in (1, 2):
            for top_groups in (1, 2, 3):
                check(l, 3, f"{T} rows, {best} of a group, {top_groups} groups", scoring=scoring, groups=4, top_groups=top_groups, group_best=best, order=T < 1000)
    for t in range(len(rows)):            # a row by itself
        check(rows[t:t + 1], 2, f"row {t}", scoring=scoring, groups=4, top_groups=2, group_best=1)


def test_groups_of_one_with_equal_scores():
    """Groups of one expert, as many as are chosen of them, logits so near to 0 that their scores are equal (2^-60 and less), and others."""
    g = torch.Generator().manual_seed(2)
    for E, k in ((64, 32), (40, 20), (300, 32)):
        big = torch.rand(300, E, generator=g) < 16.0 / E
        size = 2.0 ** torch.where(big, torch.randint(-40, 7, (300, E), generator=g), torch.randint(-90, -59, (300, E), generator=g)).float()
        l = torch.where(torch.rand(300, E, generator=g) < 0.2, -size, size)
        for scoring in ("sigmoid", "softmax"):
            check(l, k, f"{E} groups, {scoring}", scoring=scoring, groups=E, top_groups=k, group_best=1)
