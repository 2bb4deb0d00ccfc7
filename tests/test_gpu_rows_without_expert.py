"""Grouped products of an order whose last entries have no expert, without a host copy of the offsets: their rows of y stay as they were, and the rows of x that the order
names for them have no part in anything.  Every format; no expert at all, one row, a few rows of an expert, more than the kernels for few rows take at a time.  One-hot rows, so
that the results are decoded weights, exactly."""
import numpy as np
import pytest
import torch

from cases import canon_zero
from oracle import ccq_oracle as o
from paper_2507_07145_amd import binding as b
from paper_2507_07145_amd import routing, synth
from test_gpu_random_shapes import _ragged_arrays, _upload

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 5


@pytest.fixture(scope="module", params=["narrow", "wide", "mixed", "h16"])
def experts(request):
    K, N = 640, 100
    rng = synth.rng(81, len(request.param))
    gf = synth.group_format_map(K // 64, 3, rng) if request.param == "mixed" else None
    parts = [_ragged_arrays(request.param, 0, K, N, gf, rng) for _ in range(E)]
    return _upload(request.param, 0, K, N, gf, parts), [p["W"] for p in parts]


@pytest.mark.parametrize("T,k,none", [(1, 1, 1.0), (1, 2, 0.5), (2, 2, 0.5), (3, 1, 0.4), (4, 1, 1.0), (20, 2, 0.3), (150, 3, 0.2), (400, 1, 0.7)])
def test_rows_behind_the_last_expert(experts, T, k, none):
    w, W = experts
    rng = np.random.default_rng(T + k)
    ids = rng.integers(0, E, (T, k)).astype(np.int32)
    ids.reshape(-1)[rng.permutation(T * k)[:round(none * T * k)]] = -1
    order = routing.sort_rows(torch.from_numpy(ids).to(DEV), E)
    have = int(order.offsets[-1])
    assert have == (ids >= 0).sum() < T * k
    ks = rng.integers(0, w.K, T)
    x = torch.full((T + 1, w.K), float("nan"), dtype=torch.bfloat16, device=DEV)      # the last row: what the entries without an expert name
    x[:T] = b.bf16_tensor(synth.one_hot_bf16(ks, w.K), DEV)
    order.rows[have:] = T
    y = torch.full((T * k, (w.N + 7) // 8 * 8), 7.0, dtype=torch.bfloat16, device=DEV)
    b.grouped_gemm(w, x, order.rows, order.offsets, out=y[:, :w.N])
    assert bool((y[have:] == 7.0).all()) and bool((y[:, w.N:] == 7.0).all())
    rows, of = order.rows[:have].cpu().numpy(), order.experts[:have].cpu().numpy()
    want = np.stack([W[e][:, ks[t]] for t, e in zip(rows, of)]) if have else np.zeros((0, w.N))
    assert np.array_equal(canon_zero(b.bf16_bits(y[:have, :w.N])), canon_zero(o.to_bf16_bits(want)))
