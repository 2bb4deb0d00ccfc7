"""A router's choice against its definition in 64 bits: ids equal, weights within fp32's rounding."""
import numpy as np
import pytest
import torch

import routing_ref as ref
from paper_2507_07145_amd import routing

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def logits_of(T, E, seed, dtype=torch.float32, std=1.5):
    return (torch.randn(T, E, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def check_order(o, ids, experts, what, first=0):
    rows, ex, offsets, places = ref.order(ids, experts, first)
    for name, want in (("rows", rows), ("experts", ex), ("offsets", offsets), ("places", places)):
        assert np.array_equal(getattr(o, name).cpu().numpy(), want), f"{what}: {name}"


def check(l, k, what, bias=None, order=True, **kw):
    r = routing.route(l.to(DEV), k, bias=None if bias is None else bias.to(DEV), order=order, **kw)
    ids, weights = ref.route(l.double().numpy(), k, bias=None if bias is None else bias.double().numpy(), **kw)
    assert np.array_equal(r.ids.cpu().numpy(), ids), what
    # the definition's 64 bits and the kernel's, each off by some 100 steps of 2^-53, then one rounding
    ref.near(r.weights.cpu().numpy(), weights, 2.0 ** -45 * np.abs(weights) + 2.0 ** -149, what, half_step=ref.U24)
    if order:
        check_order(r.order, ids, l.shape[1], what)
    else:
        assert r.order is None
    return r


@pytest.mark.parametrize("E", [1, 2, 15, 16, 17, 64, 65, 100, 128, 129, 160, 256, 257, 500, 512, 513, 1000, 1024])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_numbers_of_experts(E, scoring):
    for T, k, dtype in ((1, min(E, 8), torch.float32), (37, min(E, 6), torch.bfloat16)):
        bias = torch.randn(E, generator=torch.Generator().manual_seed(E)) * 0.2
        for b in (None, bias):
            for renormalize in (False, True):
                check(logits_of(T, E, E + T, dtype), k, f"{T} x {E}, {k}, {scoring}, bias {b is not None}, {renormalize}", bias=b, scoring=scoring, renormalize=renormalize, scale=2.5)


@pytest.mark.parametrize("E,groups,top_groups,k", [(64, 8, 3, 8), (256, 8, 4, 8), (160, 8, 3, 6), (256, 16, 5, 8), (96, 3, 2, 32), (24, 24, 8, 8), (40, 8, 1, 5), (1024, 32, 4, 8), (1000, 10, 3, 7),
                                                   (512, 128, 9, 8), (256, 256, 8, 8)])
@pytest.mark.parametrize("best", [1, 2])
def test_groups(E, groups, top_groups, k, best):
    for scoring, with_bias, dtype in (("sigmoid", True, torch.float32), ("softmax", False, torch.bfloat16), ("sigmoid", False, torch.float32), ("softmax", True, torch.bfloat16)):
        bias = torch.randn(E, generator=torch.Generator().manual_seed(1)) * 0.1 if with_bias else None
        for T in (1, 21):
            check(logits_of(T, E, T + E, dtype), k, f"{E} in {groups}, {top_groups}, {scoring}", bias=bias, scoring=scoring, groups=groups, top_groups=top_groups, group_best=best, renormalize=True)


@pytest.mark.parametrize("k", [1, 2, 15, 16, 17, 31, 32])
def test_numbers_chosen(k):
    for E in (32, 100, 300, 1024):
        check(logits_of(19, E, k), k, f"{k} of {E}", scoring="softmax")
        check(logits_of(19, E, k), k, f"{k} of {E}", scoring="sigmoid", bias=torch.linspace(-1, 1, E), renormalize=True)


@pytest.mark.parametrize("T", [1, 3, 4, 15, 16, 17, 63, 64, 65, 200, 255, 256, 257, 1000, 5000])
def test_numbers_of_rows(T):
    check(logits_of(T, 48, T), 4, f"{T} rows", renormalize=True)
    check(logits_of(T, 48, T), 4, f"{T} rows, groups", bias=torch.linspace(-0.1, 0.1, 48), scoring="sigmoid", groups=6, top_groups=2)


def test_no_rows():
    r = routing.route(torch.empty(0, 16, device=DEV), 4)
    assert r.ids.shape == (0, 4) and r.weights.shape == (0, 4) and r.order.places.shape == (0, 4) and r.order.rows.numel() == 0
    assert r.order.offsets.tolist() == [0] * 17


def test_equal_values_go_by_the_lower_index():
    l = torch.zeros(5, 64)
    l[1, 10:20] = 1.0
    l[2] = torch.arange(64).flip(0) // 8
    l[3, ::3] = 2.0
    l[4, 63] = 5.0
    for kw in (dict(), dict(scoring="sigmoid"), dict(bias=torch.zeros(64)), dict(scoring="sigmoid", bias=torch.full((64,), 0.25)),
               dict(groups=8, top_groups=2), dict(groups=8, top_groups=2, group_best=1, bias=torch.zeros(64)), dict(groups=8, top_groups=3, scoring="sigmoid", group_best=2)):
        check(l, 8, f"ties {kw.keys()}", **kw)


def test_scores_next_to_each_other():
    """Scores plus biases that are equal in 32 bits and differ in 64: neighbours of one logit with biases that nearly make up for it."""
    E = 64
    l = torch.linspace(0.5, 0.5 + 63 * 2.0 ** -12, E).repeat(4, 1)
    l[1] = l[1].flip(0)
    l[2] = l[2][torch.randperm(E, generator=torch.Generator().manual_seed(3))]
    s = torch.sigmoid(l[0].double())
    bias = (1.0 - s).float()      # sums within 2^-25 of 1
    check(l, 8, "near sums", scoring="sigmoid", bias=bias)
    check(l, 8, "near sums in groups", scoring="sigmoid", bias=bias, groups=8, top_groups=4)


@pytest.mark.parametrize("E,k", [(64, 8), (128, 4), (256, 8), (256, 12), (256, 16), (500, 6), (1000, 32)])
@pytest.mark.parametrize("T", [6, 2100])
def test_many_rows_with_equal_and_nearly_equal_values(T, E, k):
    """Few different logits, biases of 0 or of some 2^-22: order by index, by the last bits, and among more candidates than are looked at first."""
    if T * E > 600000:
        T //= 4
    g = torch.Generator().manual_seed(E + T)
    steps = torch.randint(0, 7, (T, E), generator=g) * 0.25
    tiny = torch.randint(-8, 9, (E,), generator=g) * 2.0 ** -24
    for scoring, bias in (("sigmoid", torch.zeros(E)), ("sigmoid", tiny), ("softmax", tiny), ("softmax", None)):
        check(steps, k, f"{scoring} {bias is not None}", scoring=scoring, bias=bias, order=False, renormalize=True)
    near = 1.0 + torch.randint(0, 40, (T, E), generator=g) * 2.0 ** -23     # neighbours in fp32
    check(near, k, "neighbours", order=False)
    check(near, k, "neighbours, biased", order=False, scoring="sigmoid", bias=tiny)
    if E % 8 == 0:
        for scoring in ("sigmoid", "softmax"):
            check(steps, min(k, E // 8 * 3), "groups", order=False, scoring=scoring, bias=tiny, groups=8, top_groups=3)
            check(near, min(k, E // 8 * 3), "groups of neighbours", order=False, scoring=scoring, groups=8, top_groups=3)


def test_closed_experts():
    inf, nan = float("inf"), float("nan")
    l = logits_of(9, 40, 5)
    l[0] = -inf                            # nothing left
    l[1] = nan
    l[2, :37] = -inf                       # fewer than are asked for
    l[3, 5] = inf
    l[4, 3:6] = inf
    l[5, ::2] = nan
    l[6] = torch.finfo(torch.float32).min  # the type's lowest value is a number
    l[7] = -800.0                          # sigmoids and their sum are 0 in 64 bits
    l[8, 0] = 3e38
    bias = torch.zeros(40)
    bias[7], bias[9], bias[11], bias[38] = -inf, nan, inf, 0.5
    for scoring in ("softmax", "sigmoid"):
        for renormalize in (False, True):
            for b in (None, bias):
                check(l, 8, f"closed {scoring} {renormalize} {b is not None}", scoring=scoring, bias=b, renormalize=renormalize)
                check(l, 4, f"closed in groups {scoring} {renormalize} {b is not None}", scoring=scoring, bias=b, renormalize=renormalize, groups=10, top_groups=3)
    check(l.bfloat16(), 8, "closed bf16")


def test_rows_that_start_anywhere():
    for dtype in (torch.float32, torch.bfloat16):
        wide = logits_of(30, 203, 8, dtype)
        for view in (wide[:, 1:130], wide[::2, 3:200], wide[3:4, 7:20], wide.view(-1)[1:1 + 29 * 203].view(29, 203)[:, :77]):
            l = view.to(DEV) if view.is_contiguous() else wide.to(DEV).as_strided(view.shape, view.stride(), view.storage_offset())
            r = routing.route(l, 5)
            ids, weights = ref.route(view.double().numpy(), 5)
            assert np.array_equal(r.ids.cpu().numpy(), ids)
            ref.near(r.weights.cpu().numpy(), weights, 2.0 ** -45 * np.abs(weights), "view", half_step=ref.U24)


def test_without_order_and_on_another_stream():
    l = logits_of(50, 64, 9)
    check(l, 6, "no order", order=False)
    stream = torch.cuda.Stream()
    d = l.to(DEV)
    stream.wait_stream(torch.cuda.current_stream())
    for kw in (dict(), dict(scoring="sigmoid", groups=4, top_groups=2)):
        r = routing.route(d, 6, stream=stream, **kw)
        torch.cuda.current_stream().wait_stream(stream)
        ids, _ = ref.route(l.double().numpy(), 6, **kw)
        assert np.array_equal(r.ids.cpu().numpy(), ids)
        check_order(r.order, ids, 64, "stream")


def test_captured():
    l = logits_of(700, 64, 10).to(DEV)
    bias = torch.linspace(-0.1, 0.1, 64, device=DEV)
    call = lambda: routing.route(l, 8, scoring="sigmoid", bias=bias, groups=8, top_groups=4, renormalize=True)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = call()
    for seed in (11, 12, 13):
        l.copy_(logits_of(700, 64, seed))
        graph.replay()
        want = call()
        torch.cuda.synchronize()
        for got, w in zip((r.ids, r.weights, *r.order), (want.ids, want.weights, *want.order)):
            assert torch.equal(got, w)


@pytest.mark.parametrize("T", [3, 40, 2100])
def test_zeros_of_either_sign_are_equal(T):
    g = torch.Generator().manual_seed(T)
    l = torch.tensor([0.0, -0.0, 1.0, -1.0])[torch.randint(0, 4, (T, 64), generator=g)]
    l[0] = torch.tensor([-0.0, 0.0]).repeat(32)
    for dtype in (torch.bfloat16, torch.float32):
        for kw in (dict(), dict(scoring="sigmoid", groups=8, top_groups=3), dict(groups=8, top_groups=4, group_best=1), dict(bias=torch.zeros(64))):
            check(l.to(dtype), 30 if not kw else 8, f"{T} {dtype} {kw.keys()}", **kw)


def test_groups_of_one_and_all_experts():
    for T in (1, 8, 9):
        check(logits_of(T, 1024, T), 32, f"{T} rows, a group each", groups=1024, top_groups=40, group_best=2, bias=torch.linspace(-0.1, 0.1, 1024))
        check(logits_of(T, 1024, T), 32, f"{T} rows, two groups", groups=2, top_groups=1, scoring="sigmoid")


def test_logits_past_32_bits():
    T, E = (1 << 22) + 3, 1024
    l = torch.empty(T, E, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(1))
    r = routing.route(l, 2, renormalize=True)
    for t in (0, 1 << 21, T - 9):
        part = check(l[t:t + 9].cpu(), 2, f"from row {t}", renormalize=True)
        assert torch.equal(r.ids[t:t + 9], part.ids) and torch.equal(r.weights[t:t + 9], part.weights)
    assert torch.equal(r.order.experts[r.order.places.flatten().long()], r.ids.flatten()) and torch.equal(r.order.offsets[1:], r.ids.flatten().bincount(minlength=E).cumsum(0).int())
