"""A router, the 2-bit grouped products and the weighted sum together; and the example's layers with experts and with adapters."""
import importlib.util
import os

import pytest
import torch

from paper_2507_07145_amd import binding as ccq
from paper_2507_07145_amd import routing

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

_spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "decoder_layer.py"))


@pytest.fixture(scope="module")
def example():
    m = importlib.util.module_from_spec(_spec)
    _spec.loader.exec_module(m)
    return m


K, F, N, E = 256, 192, 320, 12


@pytest.fixture(scope="module")
def mixture(example):
    """Experts and their weights as the products decode them, rounded to bf16 (what one-hot rows give)."""
    torch.manual_seed(5)
    up = [ccq.quantize(torch.randn(2 * F, K, device=DEV) * K ** -0.5, ccq.NARROW) for _ in range(E)]
    down = [ccq.quantize(torch.randn(N, F, device=DEV) * F ** -0.5, ccq.WIDE) for _ in range(E)]
    decoded = [[ccq.gemm(w, torch.eye(w.K, device=DEV, dtype=torch.bfloat16)).double().t().contiguous() for w in kind] for kind in (up, down)]
    stacked = ccq.Weight()     # (the wide format has no alpha and beta)
    stacked.codes, stacked.scales = torch.cat([w.codes for w in down]), torch.cat([w.scales for w in down])
    stacked.desc, stacked.info, stacked.E = down[0].desc, down[0].info, E
    stacked.desc.codes, stacked.desc.scales = stacked.codes.data_ptr(), stacked.scales.data_ptr()
    return example.experts(up), stacked, decoded


def through(mixture, example, x, logits, k, shared, first=0, **kw):
    up, down, _ = mixture
    r = routing.route(logits, k, **kw)
    order = r.order
    y = ccq.grouped_gemm(up, x, order.rows, order.offsets)
    z = ccq.grouped_gemm(down, example.gated(y), torch.arange(y.shape[0], dtype=torch.int32, device=DEV), order.offsets)
    return r, routing.combine(z, order.places, r.weights, base=shared)


def expected(mixture, x, r, shared):
    _, _, (up, down) = mixture
    out = shared.double()
    for t in range(x.shape[0]):
        for e, w in zip(r.ids[t].tolist(), r.weights[t].double().tolist()):
            if e >= 0:
                y = up[e] @ x[t].double()
                out[t] += w * (down[e] @ (torch.nn.functional.silu(y[:F]) * y[F:]))
    return out


@pytest.mark.parametrize("T,k", [(1, 1), (1, 4), (3, 2), (40, 4), (200, 3), (700, 2)])
def test_a_layer_of_experts(mixture, example, T, k):
    """Against 64 bits, each token by itself.  The products round to bf16 twice and the gate once (2^-8 of a value at most), the reference's weights are rounded once for each
    product (2^-9); errors of that size in every factor change a token's sum by less than 2^-8 (3 + 1) + 2^-8 for its own rounding in norm, with room for the gate's slope
    (at most 1.1) squared.  A token at a wrong expert, place or weight is off by its whole size."""
    torch.manual_seed(T)
    x, logits = torch.randn(T, K, device=DEV).bfloat16(), torch.randn(T, E, device=DEV)
    shared = torch.randn(T, N, device=DEV).bfloat16()
    bias = torch.randn(E, device=DEV) * 0.1
    if T > 10:
        logits[T - 3:] = float("-inf")     # rows of a padded batch: no expert
        logits[5, 2:] = float("nan")       # fewer than k
    for kw in (dict(renormalize=True), dict(scoring="sigmoid", bias=bias, groups=4, top_groups=2, scale=2.5)):
        r, got = through(mixture, example, x, logits, k, shared, **kw)
        want = expected(mixture, x, r, shared)
        assert torch.isfinite(got).all()
        off = (got.double() - want).norm(dim=1) / want.norm(dim=1)
        assert off.max().item() < 6 * 2.0 ** -8, (off.max(), off.argmax())
        if T > 10:
            assert torch.equal(got[T - 3:], shared[T - 3:])
            assert int(r.order.offsets[-1]) < T * k


@pytest.mark.parametrize("T,k", [(1, 2), (2, 2), (3, 1), (20, 2)])
def test_rows_without_an_expert(mixture, example, T, k):
    """The grouped product leaves the rows behind the last expert's alone, whichever of its kernels runs (up to four rows, more)."""
    up, _, _ = mixture
    torch.manual_seed(T)
    x, logits = torch.randn(T, K, device=DEV).bfloat16(), torch.randn(T, E, device=DEV)
    logits[0, 1:] = float("-inf")      # one expert, and none in the place after it
    logits[T // 2 + 1:] = float("-inf")
    o = routing.route(logits, k).order
    have = int(o.offsets[-1])
    assert have < T * k
    y = torch.full((T * k, 2 * F), 7.0, dtype=torch.bfloat16, device=DEV)
    ccq.grouped_gemm(up, x, o.rows, o.offsets, out=y)
    assert bool((y[have:] == 7.0).all())
    for p in range(have):
        w = mixture[2][0][int(o.experts[p])]
        want = w @ x[int(o.rows[p])].double()
        assert ((y[p].double() - want).norm() / want.norm()).item() < 3 * 2.0 ** -8   # (rounding of the result, of the reference's weights)


def test_a_share_of_the_experts(mixture, example):
    """Two GPUs' shares of the experts, one after the other, add up to all of them."""
    up, down, _ = mixture
    T, k, half = 90, 3, E // 2
    torch.manual_seed(9)
    x, logits = torch.randn(T, K, device=DEV).bfloat16(), torch.randn(T, E, device=DEV)
    none = torch.zeros(T, N, device=DEV)
    r, _ = through(mixture, example, x, logits, k, none, renormalize=True)
    total = none.clone()
    for first in (0, half):
        share = []
        for w in (up, down):
            part = ccq.Weight()
            for n in ("codes", "scales", "alpha", "beta"):
                v = getattr(w, n)
                setattr(part, n, None if v is None else v[first:first + half].contiguous())
            d = part.desc = type(w.desc).from_buffer_copy(w.desc)
            part.info, part.E = w.info, half
            d.codes, d.scales = part.codes.data_ptr(), part.scales.data_ptr()
            d.code_alpha, d.code_beta = (None if t is None else t.data_ptr() for t in (part.alpha, part.beta))
            share.append(part)
        o = routing.sort_rows(r.ids, half, first=first)
        y = ccq.grouped_gemm(share[0], x, o.rows, o.offsets)
        z = ccq.grouped_gemm(share[1], example.gated(y), torch.arange(T * k, dtype=torch.int32, device=DEV), o.offsets)
        routing.combine(z, o.places, r.weights, base=total, out=total)
    want = expected(mixture, x, r, none)
    assert ((total.double() - want).norm(dim=1) / want.norm(dim=1)).max().item() < 6 * 2.0 ** -8


@pytest.mark.parametrize("kind", [dict(experts=8, top_k=3), dict(adapters=2, rank=16), dict(experts=6, top_k=2, adapters=3, rank=8)])
def test_a_replayed_graph_gives_the_eager_steps(example, kind):
    n, steps, count = 61, 6, 5
    torch.manual_seed(3)
    decoder = example.Decoder(layers=2, hidden=512, heads=8, kv_heads=2, feed_forward=256, sequences=count, room=200, **kind)
    prompt = torch.randn(count * n, 512, device="cuda").bfloat16()
    xs = torch.randn(steps, count, 512, device="cuda").bfloat16()

    def start():
        decoder.state.lens.zero_()
        assert torch.isfinite(decoder.prompt(prompt)).all()

    start()
    eager = [decoder.token(x).clone() for x in xs]
    start()
    x = xs[0].clone()
    graph, y = example.capture(decoder, x)
    start()
    for i in range(steps):
        x.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), eager[i].view(torch.int16)), i
        torch.randn(1 << 16, device="cuda").sum().item()   # eager work of the program between replays


def test_adapters_of_sequences(example):
    """A sequence with an adapter gives what it gives in a batch of its own, one without gives what a model without adapters gives; the adapter's part is there.  The kernels of
    another number of rows add in another order, and where that changes an 8-bit value it is by 2^-4 of it: the bound of two such layers."""
    n, count = 30, 3
    torch.manual_seed(4)
    decoder = example.Decoder(layers=2, hidden=512, heads=8, kv_heads=2, feed_forward=512, sequences=count, room=64, adapters=2, rank=16)
    x = torch.randn(count * n, 512, device="cuda").bfloat16()
    whole = decoder.prompt(x).view(count, n, 512).float()
    decoder.state.lens.zero_()
    decoder.state.adapter.fill_(-1)
    plain = decoder.prompt(x).view(count, n, 512).float()
    decoder.state.lens.zero_()
    decoder.state.adapter.fill_(1)
    second = decoder.prompt(x).view(count, n, 512).float()
    near = lambda a, b: ((a - b).norm() / b.norm()).item() < 2 * 2.0 ** -4  # noqa: E731
    assert near(whole[0], plain[0]) and near(whole[2], second[2])       # sequences 0, 1, 2 have no adapter, the first, the second
    assert not torch.equal(whole[1], plain[1]) and not torch.equal(whole[1], second[1])
