"""Pages whose scales of values lie further apart than fp32's exponents reach in one product: a page of zeros or of tiny values beside a huge one still counts in the
sum of weights."""
import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[0, 1], ids=["few", "many"], autouse=True)
def kernel(request):
    layer._load().ccq_attention_force(request.param)
    yield
    layer._load().ccq_attention_force(-1)


@pytest.mark.parametrize("big,small", [(60, -60), (58, -60), (60, -30), (20, -60), (-10, -60), (-60, -60)])
@pytest.mark.parametrize("below", [0, 6, 10, 40])
@pytest.mark.parametrize("pairs", [[(1, 4000)], [(40, 3000)]], ids=["one", "chunk"])
@pytest.mark.parametrize("P,D", [(16, 128), (64, 128), (32, 64)])
def test_a_huge_page_among_tiny_ones(big, small, below, pairs, P, D):
    """The huge page's tokens have scores `below` (in units of log 2) above the others'."""
    seq = r.Sequences(pairs, P, 1)
    cache = r.random_cache(seq, 1, D, 2)
    page = int(seq.table[0, 5])
    g = r.gen(3)
    # keys: 0 in the huge page; elsewhere the first dimension takes the score down, the second spreads it
    cache[0][:] = torch.zeros(cache[0].shape).to(r.E4M3).view(torch.uint8)
    cache[0][..., 0] = torch.full(cache[0].shape[:-1], -1.0).to(r.E4M3).view(torch.uint8)
    cache[0][..., 1] = torch.randn(cache[0].shape[:-1], generator=g).clamp(-3, 3).to(r.E4M3).view(torch.uint8)
    cache[0][page] = 0
    cache[2][:], cache[3][:] = 127, 127 + small
    cache[3][page] = 127 + big
    q = torch.zeros(seq.T, 2, D)
    q[..., 0], q[..., 1] = below, 1.0
    q = q.bfloat16()
    scale = 0.6931471805599453
    got = layer.attention(r.to_device(cache), seq.batch(), q.to(r.DEV), scale=scale).cpu().double()
    want, size = r.attend(seq, cache, q, scale)
    assert bool(((got - want).abs() <= r.attend_limit(want, size)).all()), float(((got - want).abs() / r.attend_limit(want, size)).max())
