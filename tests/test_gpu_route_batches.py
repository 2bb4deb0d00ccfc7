"""A row's choice is the row's own: the same whatever else the batch holds and however many rows it has, where two sums differ in their last bit too."""
import numpy as np
import pytest
import torch

from paper_2507_07145_amd import routing
from test_gpu_route import logits_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

PLACES = (0, 17, 34, 51)   # in four lanes and four values of a lane


def near_sums(n, seed):
    """n rows of 64 logits, four open, and their biases: the sums of the first two are equal to some steps of 2^-54.  exp(l0 - l2) - exp(l1 - l2) = b1 total is solved for the
    total: l2 coarsely, then the fourth's small part."""
    rng = np.random.default_rng(seed)
    beta = 2.0 ** -25
    rows = np.full((n, 64), -np.inf, dtype=np.float32)
    have = 0
    while have < n:
        l0 = np.float32(rng.uniform(-1, 1))
        l1 = np.float32(l0 - rng.integers(1, 6) * 2.0 ** -24)
        tops = np.float32(l0 + np.linspace(0.0, 3.0, 4001))
        p0, p1 = np.exp(np.float64(l0) - tops), np.exp(np.float64(l1) - tops)
        part = (p0 - p1) / beta - (1.0 + p0 + p1)
        fits = np.nonzero((part > 2.0 ** -40) & (part < 2.0 ** -9))[0]
        if len(fits) == 0:
            continue
        i = fits[rng.integers(len(fits))]
        rows[have, list(PLACES)] = l0, l1, tops[i], np.float32(tops[i] + np.log(part[i]))
        have += 1
    bias = np.zeros(64, dtype=np.float32)
    bias[list(PLACES)] = 0.0, beta, -1.0, -1.0
    return torch.from_numpy(rows), torch.from_numpy(bias)


def test_the_same_choice_in_any_batch():
    """Sums of softmax scores and biases that differ in their last bits: the choice is the row's own, whatever else the batch holds and however many rows it has."""
    n = 1024
    rows, bias = near_sums(n, 1)
    clear, equal = torch.linspace(-3, 3, 64), torch.zeros(64)
    results = []
    for filler in (clear, equal):        # neighbours that leave no doubt, and such as are chosen on 64 bits throughout
        l = filler.repeat(4 * n, 1)
        l[::4] = rows
        r = routing.route(l.to(DEV), 1, bias=bias.to(DEV), order=False)
        results.append((r.ids[::4].cpu(), r.weights[::4].cpu()))
    for T in (n, 8):                     # a wavefront for each row, and with the order in one launch
        parts = [routing.route(rows[t:t + T].to(DEV), 1, bias=bias.to(DEV)) for t in range(0, n, T)]
        results.append((torch.cat([p.ids for p in parts]).cpu(), torch.cat([p.weights for p in parts]).cpu()))
    ids, weights = results[0]
    counts = ids.flatten().bincount(minlength=64)
    assert min(int(counts[0]), int(counts[17])) > n // 20 and int(counts[0] + counts[17]) == n     # (the sums are that near)
    for i, (other, w) in enumerate(results[1:]):
        assert torch.equal(other, ids), f"batch {i + 1}: {int((other != ids).sum())} rows"
        assert torch.equal(w, weights)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_the_same_weights_in_any_batch(scoring):
    l = logits_of(2300, 160, 4)
    bias = torch.linspace(-0.1, 0.1, 160).to(DEV)
    for k, kw in ((20, dict(renormalize=True)), (31, dict(bias=bias)), (6, dict(bias=bias, groups=8, top_groups=3, renormalize=True, scale=2.5))):
        whole = routing.route(l.to(DEV), k, scoring=scoring, order=False, **kw)
        for n in (1150, 5):
            part = routing.route(l[:n].to(DEV), k, scoring=scoring, **kw)
            assert torch.equal(part.ids, whole.ids[:n]) and torch.equal(part.weights, whole.weights[:n])
