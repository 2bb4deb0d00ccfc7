"""The example's classes take their arguments in the order that they had before experts and adapters came."""
import pytest
import torch

from test_gpu_mixture import example  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_the_device_comes_before_experts_and_adapters(example):  # noqa: F811
    made = []
    for args, kw in (((2, 512, 8, 2, 512, 2, 64, "cuda:0"), {}), ((2, 512, 8, 2, 512, 2, 64), {})):
        torch.manual_seed(7)
        decoder = example.Decoder(*args, **kw)
        made.append(decoder.token(torch.randn(2, 512, device="cuda").bfloat16()).clone())
    assert torch.equal(*made) and bool(made[0].isfinite().all())
    assert example.Sequences(2, 100, "cuda:0").order(1) is None and example.Sequences(4, 100, "cuda:0", 3).adapter.tolist() == [-1, 0, 1, 2]
