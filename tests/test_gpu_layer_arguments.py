"""Arguments of the layer operators on the GPU: what the native path and the general one make of them is the same."""
import pytest
import torch

import layer_ref as r
from paper_2507_07145_amd import layer

pytestmark = pytest.mark.gpu


def test_scales_whose_rows_share_memory_are_refused():
    w = layer.Weight8(torch.zeros(64, 256, dtype=torch.uint8, device=r.DEV), torch.ones(1, 2, device=r.DEV))
    codes, one = torch.zeros(4, 256, dtype=torch.uint8, device=r.DEV), torch.full((1, 2), 127, dtype=torch.uint8, device=r.DEV)
    for kw in ({}, dict(stream=torch.cuda.current_stream())):
        with pytest.raises((ValueError, layer.CcqError)):
            layer.gemm8(w, layer.Rows8(codes, one.expand(4, 2)), **kw)
    assert layer.gemm8(w, layer.Rows8(codes, one.repeat(4, 1))).shape == (4, 64)
