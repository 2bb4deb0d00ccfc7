"""The weighted sum of the experts' rows against 64 bits."""
import numpy as np
import pytest
import torch

import routing_ref as ref
from paper_2507_07145_amd import routing

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(T, k, N, P, seed, none=0.2):
    g = torch.Generator().manual_seed(seed)
    rows = torch.randn(P, N, generator=g).bfloat16()
    places = torch.randint(0, max(P, 1), (T, k), generator=g, dtype=torch.int32)
    places[torch.rand(T, k, generator=g) < none] = -1
    return rows, places, torch.randn(T, k, generator=g), torch.randn(T, N, generator=g)


def check(rows, places, weights, base, got, what):
    want, off = ref.combine(rows.double().numpy(), places.numpy(), weights.double().numpy(), None if base is None else base.double().numpy())
    ref.near(got.double().cpu().numpy(), want, off, what, half_step=ref.U24 if got.dtype == torch.float32 else ref.U8)


@pytest.mark.parametrize("N", [1, 7, 8, 9, 500, 511, 512, 513, 1000, 4096])
@pytest.mark.parametrize("T,k", [(1, 1), (1, 8), (5, 2), (33, 6), (3, 9), (2, 32)])
def test_sizes(N, T, k):
    rows, places, weights, base = inputs(T, k, N, T * k + 3, N + T)
    d = lambda t: t.to(DEV)  # noqa: E731
    check(rows, places, weights, None, routing.combine(d(rows), d(places), d(weights)), "no base")
    b16 = base.bfloat16()
    check(rows, places, weights, b16, routing.combine(d(rows), d(places), d(weights), base=d(b16)), "bf16 base")
    check(rows, places, weights, base, routing.combine(d(rows), d(places), d(weights), base=d(base)), "fp32 base")
    out = torch.empty(T, N, device=DEV)
    assert routing.combine(d(rows), d(places), d(weights), base=d(b16), out=out) is out
    check(rows, places, weights, b16, out, "fp32 out")
    total = d(base)
    routing.combine(d(rows), d(places), d(weights), base=total, out=total)   # in place
    check(rows, places, weights, base, total, "in place")


def test_places_out_of_range_and_what_they_hide():
    """Places outside the rows are left out with their weights, whatever these are; rows of no place are not looked at."""
    rows, places, weights, base = inputs(6, 4, 100, 10, 1, none=0.0)
    places[0] = torch.tensor([-1, 10, 2 ** 31 - 1, -2 ** 31])
    weights[0] = torch.tensor([float("nan"), float("inf"), 1.0, 2.0])
    places[1] = torch.tensor([3, 3, 3, -1])     # the same row twice
    places[places == 7] = 6
    rows[7] = float("nan")
    check(rows, places, weights, None, routing.combine(rows.to(DEV), places.to(DEV), weights.to(DEV)), "out of range")
    check(rows, places, weights, base, routing.combine(rows.to(DEV), places.to(DEV), weights.to(DEV), base=base.to(DEV)), "out of range, base")
    assert not bool(routing.combine(rows[:0].to(DEV), places.to(DEV), weights.to(DEV)).any())   # no rows at all


def test_nan_and_infinities_stay_in_their_tokens():
    rows, places, weights, _ = inputs(4, 2, 64, 8, 2, none=0.0)
    places[:] = torch.arange(8, dtype=torch.int32).view(4, 2)
    weights.abs_().add_(0.5)
    rows[2, 5], rows[4, 6], rows[5, 6], rows[6, 7] = float("nan"), float("inf"), -float("inf"), float("inf")
    with np.errstate(invalid="ignore"):
        want, off = ref.combine(rows.double().numpy(), places.numpy(), weights.double().numpy())
    ref.near(routing.combine(rows.to(DEV), places.to(DEV), weights.to(DEV)).double().cpu().numpy(), want, np.nan_to_num(off), "specials")


def test_strides_and_stream():
    rows, places, weights, base = (t.to(DEV) for t in inputs(40, 10, 703, 90, 3))
    r, p, w, b = rows[::2, 3:300], places[:, 1:7], weights[:, 2:8], base[:, 5:302]
    p = torch.where(p >= r.shape[0], -1, p)
    out = torch.full((40, 400), 9.0, dtype=torch.bfloat16, device=DEV)
    routing.combine(r, p, w, base=b, out=out[:, 1:298])
    check(r.cpu(), p.cpu(), w.cpu(), b.cpu(), out[:, 1:298], "views")
    assert bool((out[:, :1] == 9).all()) and bool((out[:, 298:] == 9).all())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = routing.combine(r, p, w, base=b, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, out[:, 1:298])


def test_far_rows():
    """Rows past 2^31 elements."""
    N = 4096
    rows = torch.empty(530000, N, dtype=torch.bfloat16, device=DEV)
    places = torch.tensor([[529999, 0], [524288, 300000]], dtype=torch.int32, device=DEV)
    rows[places.flatten().long()] = torch.randn(4, N, device=DEV).bfloat16()
    weights = torch.randn(2, 2, device=DEV)
    got = routing.combine(rows, places, weights)
    check(rows[places.flatten().long()].cpu(), torch.arange(4).view(2, 2), weights.cpu(), None, got, "far rows")


def test_captured():
    rows, places, weights, base = (t.to(DEV) for t in inputs(20, 8, 1000, 160, 4))
    routing.combine(rows, places, weights, base=base)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = routing.combine(rows, places, weights, base=base)
    for seed in (5, 6, 7):
        for t, n in zip((rows, places, weights, base), inputs(20, 8, 1000, 160, seed)):
            t.copy_(n)
        graph.replay()
        assert torch.equal(y, routing.combine(rows, places, weights, base=base))


def test_rows_past_32_bits():
    P, N = (1 << 19) + 5, 8200          # 4.3e9 values
    rows = torch.zeros(P, N, dtype=torch.bfloat16, device=DEV)
    rows[P - 1], rows[1 << 18], rows[3] = 3.0, 5.0, 0.5
    places = torch.tensor([[P - 1, 3], [1 << 18, P - 1], [-1, P]], dtype=torch.int32, device=DEV)
    weights = torch.tensor([[1.0, 2.0], [1.0, 0.25], [1.0, 1.0]], device=DEV)
    got = routing.combine(rows, places, weights)
    assert torch.equal(got, torch.tensor([[4.0], [5.75], [0.0]], device=DEV).bfloat16().expand(3, N))
    T = P
    places = torch.full((T, 1), 3, dtype=torch.int32, device=DEV)
    weights = (torch.arange(T, device=DEV) % 128).float()[:, None]
    got = routing.combine(rows, places, weights, base=rows)
    want = weights[:, 0] * 0.5 + rows[:, 0].float()
    for c in (0, 511, 4096, N - 1):
        assert torch.equal(got[:, c].float(), want)
