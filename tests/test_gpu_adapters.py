"""Low-rank adapters of a batch's requests against 64 bits."""
import numpy as np
import pytest
import torch

import routing_ref as ref
from paper_2507_07145_amd import routing

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Case:
    def __init__(self, T, K, N, R, n, seed, ranks=False, none=0.2, runs=0):
        g = torch.Generator().manual_seed(seed)
        self.x, self.y = torch.randn(T, K, generator=g).bfloat16(), torch.randn(T, N, generator=g).bfloat16()
        self.a, self.b = (torch.randn(n, R, K, generator=g) * K ** -0.5).bfloat16(), torch.randn(n, N, R, generator=g).bfloat16()
        self.scales = torch.rand(n, generator=g) + 0.5
        self.ranks = torch.randint(0, R + 1, (n,), generator=g, dtype=torch.int32) if ranks else None
        self.ids = torch.randint(0, n, (T,), generator=g, dtype=torch.int32)
        if runs:
            self.ids = self.ids[:runs].repeat_interleave(-(-T // runs))[:T].clone()
        self.ids[torch.rand(T, generator=g) < none] = -1
        if self.ranks is not None:   # what lies behind the ranks in use may hold anything
            for i, r in enumerate(self.ranks.tolist()):
                self.a[i, r:], self.b[i, :, r:] = float("nan"), float("inf")

    def set(self):
        d = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        return routing.Adapters(d(self.a), d(self.b), scales=d(self.scales), ranks=d(self.ranks))

    def order(self):
        return routing.sort_rows(self.ids.to(DEV)[:, None], self.a.shape[0])

    def check(self, got, what):
        f = lambda t: None if t is None else t.double().numpy()  # noqa: E731
        a, b = (np.where(np.isfinite(f(t)), f(t), 0.0) for t in (self.a, self.b))
        want, off = ref.adapters(f(self.y), f(self.x), a, b, self.ids.tolist(), f(self.scales), None if self.ranks is None else self.ranks.tolist())
        ref.near(got.double().cpu().numpy(), want, off, what)
        none = self.ids < 0
        assert torch.equal(got.cpu()[none].view(torch.int16), self.y[none].view(torch.int16)), f"{what}: rows without an adapter"


@pytest.mark.parametrize("R", [8, 16, 24, 32, 40, 64, 72, 128, 136, 256])
@pytest.mark.parametrize("T,n", [(1, 1), (1, 5), (3, 2), (16, 1), (17, 30), (64, 8), (300, 3), (290, 100)])
def test_ranks_and_rows(R, T, n):
    for ranks in (False, True):
        c = Case(T, 328, 213, R, n, R + T + n, ranks=ranks)
        c.check(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order()), f"rank {R}, {T} rows, {n} adapters, {ranks}")


@pytest.mark.parametrize("K", [8, 24, 32, 40, 256, 264, 1000, 2048, 8200])
@pytest.mark.parametrize("N", [1, 15, 16, 17, 63, 64, 65, 256, 257, 600])
def test_shapes(K, N):
    for T, n, R in ((2, 2, 16), (40, 4, 32)):
        c = Case(T, K, N, R, n, K + N + T)
        c.check(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order()), f"{T} x {K} to {N}")


@pytest.mark.parametrize("T,n,R,runs", [(1000, 4, 64, 6), (2100, 2, 16, 3), (700, 64, 128, 0), (513, 3, 256, 9), (1024, 500, 8, 0)])
def test_prompts(T, n, R, runs):
    c = Case(T, 1032, 520, R, n, T, ranks=True, runs=runs)
    c.check(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order()), f"{T} rows, {n} adapters of {R}")


def test_in_place_and_out():
    for T, R in ((5, 16), (400, 64)):
        c = Case(T, 264, 300, R, 4, T)
        y, want = c.y.to(DEV), routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order())
        assert torch.equal(y, c.y.to(DEV))
        out = torch.empty_like(y)
        assert routing.adapters(y, c.x.to(DEV), c.set(), c.order(), out=out) is out and torch.equal(out, want)
        assert routing.adapters(y, c.x.to(DEV), c.set(), c.order(), out=y) is y and torch.equal(y, want)


def test_no_scales_and_no_adapters_in_use():
    c = Case(20, 64, 48, 8, 3, 1)
    c.scales = None
    c.check(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order()), "no scales")
    c.ids[:] = -1
    c.check(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order()), "none in use")
    y = c.y.to(DEV)
    routing.adapters(y, c.x.to(DEV), c.set(), c.order(), out=y)
    assert torch.equal(y.cpu(), c.y)
    empty = routing.adapters(y[:0], c.x.to(DEV)[:0], c.set(), routing.sort_rows(torch.empty(0, 1, dtype=torch.int32, device=DEV), 3))
    assert empty.shape == (0, 48)


def test_orders_that_are_not_sorted():
    """Any permutation of the rows is right; adapters and rows outside their range are none."""
    c = Case(100, 72, 90, 16, 5, 2)
    perm = torch.randperm(100, generator=torch.Generator().manual_seed(1))
    order = routing.Order(perm.int().to(DEV), c.ids[perm].to(DEV), None, None)
    c.check(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), order), "unsorted")
    experts = c.ids[perm].clone()
    experts[3], experts[50], experts[51] = 5, 2 ** 31 - 1, -2 ** 31
    c.ids[perm[[3, 50, 51]]] = -1
    c.check(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), routing.Order(perm.int().to(DEV), experts.to(DEV), None, None)), "adapters out of range")
    rows = perm.int().clone()
    rows[7], rows[8] = 100, -1
    out = torch.zeros(100, 90, dtype=torch.bfloat16, device=DEV)
    routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), routing.Order(rows.to(DEV), experts.to(DEV), None, None), out=out)
    assert not bool(out[perm[[7, 8]]].any())
    out[perm[[7, 8]]] = routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order())[perm[[7, 8]]]
    c.check(out, "rows out of range")


def test_nan_and_infinities_stay_in_their_rows():
    for T in (40, 300):
        c = Case(T, 136, 80, 16, 3, 3, none=0.0)
        c.x[5, 7], c.x[9, 0], c.y[11, 3] = float("nan"), float("inf"), float("nan")
        got = routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order()).cpu()
        assert bool(got[5].isnan().all()) and not bool(got[9].isfinite().any()) and bool(got[11, 3].isnan()) and bool(got[11, :3].isfinite().all())
        for t in (5, 9, 11):
            c.x[t] = 0
            c.y[t] = 0
            got[t] = 0
        c.check(got, "specials")
        c.b[:] = c.b.abs()
        c.a[:] = c.a.abs()
        c.x[6, 1] = float("inf")        # infinite v, positive b: infinity, not NaN
        assert bool(torch.isposinf(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order())[6]).all())


def test_strides_and_stream():
    c = Case(60, 128, 100, 24, 6, 4, ranks=True)
    wide_x, wide_y = torch.randn(60, 300, device=DEV).bfloat16(), torch.randn(60, 333, device=DEV).bfloat16()
    wide_x[:, 5:133], wide_y[:, 7:107] = c.x.to(DEV), c.y.to(DEV)
    before = wide_y.clone()
    routing.adapters(wide_y[:, 7:107], wide_x[:, 5:133], c.set(), c.order(), out=wide_y[:, 7:107])
    c.check(wide_y[:, 7:107], "columns of wider rows")
    before[:, 7:107] = wide_y[:, 7:107]
    assert torch.equal(before, wide_y)
    one = Case(1, 128, 100, 24, 6, 4)
    one.check(routing.adapters(one.y.to(DEV), one.x.to(DEV), one.set(), one.order()), "one row")
    stream = torch.cuda.Stream()
    adapters, order, x, y = c.set(), c.order(), c.x.to(DEV), c.y.to(DEV)
    stream.wait_stream(torch.cuda.current_stream())
    got = routing.adapters(y, x, adapters, order, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, wide_y[:, 7:107])


def test_the_same_bits_every_time():
    c = Case(333, 2056, 700, 64, 7, 5)
    adapters, order, x, y = c.set(), c.order(), c.x.to(DEV), c.y.to(DEV)
    want = routing.adapters(y, x, adapters, order)
    for _ in range(5):
        assert torch.equal(routing.adapters(y, x, adapters, order), want)


@pytest.mark.parametrize("T", [4, 600])
def test_captured(T):
    c = Case(T, 1032, 520, 32, 6, 6)
    adapters, x, y, ids = c.set(), c.x.to(DEV), c.y.to(DEV), c.ids.to(DEV)[:, None]
    call = lambda: routing.adapters(y, x, adapters, routing.sort_rows(ids, 6))  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for seed in (7, 8, 9):
        n = Case(T, 1032, 520, 32, 6, seed)
        for t, v in ((x, n.x), (y, n.y), (ids, n.ids[:, None]), (adapters.a, n.a), (adapters.b, n.b)):
            t.copy_(v)
        graph.replay()
        assert torch.equal(out, call())


def test_two_calls_with_workspaces_of_their_own():
    c = Case(50, 2056, 300, 16, 6, 10)
    adapters, order, x, y = c.set(), c.order(), c.x.to(DEV), c.y.to(DEV)
    need = routing.adapters_workspace_bytes(adapters, 50)
    ws = torch.full((need + 64,), 0xAB, dtype=torch.uint8, device=DEV)
    got = routing.adapters(y, x, adapters, order, workspace=ws)
    c.check(got, "given workspace")
    assert bool((ws[need:] == 0xAB).all())
    with pytest.raises(routing.CcqError):
        routing.adapters(y, x, adapters, order, workspace=ws[:need - 16])


@pytest.mark.parametrize("T,N,n,R,runs", [(600, 7001, 4, 16, 0), (600, 7000, 6, 64, 5), (1300, 3333, 9, 128, 0), (520, 8100, 3, 256, 7), (8100, 520, 50, 32, 90), (2100, 2001, 2, 64, 3),
                                          (2050, 2056, 3, 24, 0), (4096, 1025, 600, 8, 0), (5000, 841, 1, 136, 1), (4200, 1000, 40, 72, 33)])
def test_many_rows_and_columns(T, N, n, R, runs):
    c = Case(T, 264, N, R, n, T, ranks=True, runs=runs)
    c.check(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order()), f"{T} rows to {N}, {n} adapters of {R}")


@pytest.mark.parametrize("T,N", [(900, 4701), (4500, 945)])
def test_many_in_views_and_any_order(T, N):
    """In place in columns of wider rows, in an order that is not sorted and has places that are no rows."""
    c = Case(T, 136, N, 40, 5, T, ranks=True)
    wide_x, wide_y = torch.randn(T, 150, device=DEV).bfloat16(), torch.randn(T, N + 22, device=DEV).bfloat16()
    wide_x[:, 5:141], wide_y[:, 3:3 + N] = c.x.to(DEV), c.y.to(DEV)
    before = wide_y.clone()
    perm = torch.randperm(T, generator=torch.Generator().manual_seed(T))
    rows, experts = perm.int().clone(), c.ids[perm].clone()
    rows[7], rows[800], rows[801] = T, -1, 2 ** 31 - 1
    experts[3], experts[50], experts[51] = 5, 2 ** 31 - 1, -2 ** 31
    c.ids[perm[[3, 50, 51, 7, 800, 801]]] = -1
    routing.adapters(wide_y[:, 3:3 + N], wide_x[:, 5:141], c.set(), routing.Order(rows.to(DEV), experts.to(DEV), None, None), out=wide_y[:, 3:3 + N])
    c.check(wide_y[:, 3:3 + N], "any order")
    before[:, 3:3 + N] = wide_y[:, 3:3 + N]
    assert torch.equal(before, wide_y)


def test_many_rows_specials():
    c = Case(700, 72, 6100, 16, 3, 3, none=0.0)
    c.x[5, 7], c.x[9, 0], c.y[11, 3] = float("nan"), float("inf"), float("nan")
    got = routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order()).cpu()
    assert bool(got[5].isnan().all()) and not bool(got[9].isfinite().any()) and bool(got[11, 3].isnan()) and bool(got[11, :3].isfinite().all())
    for t in (5, 9, 11):
        c.x[t], c.y[t], got[t] = 0, 0, 0
    c.check(got, "specials")
    c.a[:], c.b[:] = c.a.abs(), c.b.abs()
    c.x[6, 1] = float("inf")
    assert bool(torch.isposinf(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order())[6]).all())


def test_many_rows_captured():
    c = Case(640, 264, 6600, 32, 6, 6)
    adapters, x, y, ids = c.set(), c.x.to(DEV), c.y.to(DEV), c.ids.to(DEV)[:, None]
    call = lambda: routing.adapters(y, x, adapters, routing.sort_rows(ids, 6))  # noqa: E731
    want = call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for seed in (7, 8, 9):
        n = Case(640, 264, 6600, 32, 6, seed)
        for t, v in ((x, n.x), (y, n.y), (ids, n.ids[:, None]), (adapters.a, n.a), (adapters.b, n.b)):
            t.copy_(v)
        graph.replay()
        want = call()
        assert torch.equal(out, want)
        assert torch.equal(call(), want)


@pytest.mark.parametrize("T,N", [(3, 40), (60, 40), (700, 6100)])
def test_an_infinite_scale_stays_with_the_ranks_in_use(T, N):
    c = Case(T, 64, N, 16, 2, 5, none=0.0)
    c.a, c.b, c.x = c.a.abs(), c.b.abs() + 0.5, c.x.abs() + 0.5
    c.ranks = torch.tensor([5, 16], dtype=torch.int32)
    c.ids[:] = 0
    c.scales[0] = float("inf")
    assert bool(torch.isposinf(routing.adapters(c.y.to(DEV), c.x.to(DEV), c.set(), c.order())).all())


@pytest.mark.parametrize("T,N", [((1 << 18) + 40, 16400), ((1 << 22) + 40, 1032)])
def test_rows_past_32_bits(T, N):
    """4.3e9 results; x past 32 bits too where there are more rows than one kernel's limit."""
    K, R, n = 1032 if T > 1 << 22 else 64, 8, 3
    x, y = (torch.empty(T, c, dtype=torch.bfloat16, device=DEV) for c in (K, N))
    g = torch.Generator(DEV).manual_seed(T)
    x.normal_(generator=g), y.normal_(generator=g)
    ids = (torch.arange(T, device=DEV) % 4 - 1).int()[:, None]
    c = Case(1, K, N, R, n, 1)
    got = routing.adapters(y, x, c.set(), routing.sort_rows(ids, n))
    for t in (0, T // 2, T - 40):
        c.x, c.y, c.ids = x[t:t + 40].cpu(), y[t:t + 40].cpu(), ids[t:t + 40, 0].cpu()
        c.check(got[t:t + 40], f"from row {t}")
