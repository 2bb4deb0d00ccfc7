"""The example's layers with adapters, bit for bit: a sequence's rows go by its own adapter, whatever the others have."""
import torch

import pytest

from test_gpu_mixture import example  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_each_sequence_has_its_own(example):  # noqa: F811
    """Three runs of the same rows through the same kernels, which share no sums between rows: with an adapter each, with none, all with the second."""
    n, count = 30, 3
    torch.manual_seed(4)
    decoder = example.Decoder(layers=2, hidden=512, heads=8, kv_heads=2, feed_forward=512, sequences=count, room=64, adapters=2, rank=16)
    x = torch.randn(count * n, 512, device="cuda").bfloat16()

    def run(*adapter):
        decoder.state.lens.zero_()
        decoder.state.adapter.copy_(torch.tensor(adapter, dtype=torch.int32))
        return decoder.prompt(x).view(count, n, 512).clone()
    own, none, second = run(-1, 0, 1), run(-1, -1, -1), run(1, 1, 1)
    assert torch.equal(own[0], none[0]) and torch.equal(own[2], second[2])
    assert torch.equal(run(1, 0, -1)[1], own[1])
    for a in (none, second):
        assert not torch.equal(own[1], a[1])
    for t in range(count):     # (and an adapter is no small matter: every token is another)
        assert bool((none[t] != second[t]).any(1).all())
