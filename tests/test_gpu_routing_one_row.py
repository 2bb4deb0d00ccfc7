"""In place with a single row, whose stride may be anything: two views of one row that differ in it are the same row."""
import pytest
import torch

from paper_2507_07145_amd import routing

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def views(n, dtype):
    wide = torch.randn(1, n + 36, device=DEV).to(dtype)
    return wide, wide[:, :n], wide.as_strided((1, n), (n, 1))


@pytest.mark.parametrize("on_stream", [False, True])     # the native path, the general one
def test_strides_of_one_row(on_stream):
    stream = torch.cuda.current_stream() if on_stream else None
    g = torch.Generator(DEV).manual_seed(3)
    rows, places, weights = torch.randn(3, 64, device=DEV, generator=g).bfloat16(), torch.tensor([[2, 0]], dtype=torch.int32, device=DEV), torch.rand(1, 2, device=DEV, generator=g)
    for dtype in (torch.bfloat16, torch.float32):
        for a, b in ((1, 2), (2, 1)):
            v = views(64, dtype)
            want = routing.combine(rows, places, weights, base=v[a].clone(), out=torch.empty(1, 64, dtype=dtype, device=DEV))
            rest = v[0][:, 64:].clone()
            assert routing.combine(rows, places, weights, base=v[a], out=v[b], stream=stream) is v[b]
            assert torch.equal(v[a], want) and torch.equal(v[0][:, 64:], rest)
    adapters = routing.Adapters(torch.randn(2, 8, 32, device=DEV, generator=g).bfloat16(), torch.randn(2, 64, 8, device=DEV, generator=g).bfloat16())
    x, order = torch.randn(1, 32, device=DEV, generator=g).bfloat16(), routing.sort_rows(torch.ones(1, 1, dtype=torch.int32, device=DEV), 2)
    for a, b in ((1, 2), (2, 1)):
        v = views(64, torch.bfloat16)
        want = routing.adapters(v[a].clone(), x, adapters, order)
        rest = v[0][:, 64:].clone()
        routing.adapters(v[a], x, adapters, order, out=v[b], stream=stream)
        assert torch.equal(v[a], want) and torch.equal(v[0][:, 64:], rest)
