"""The refusals of the operators around rows that choose their weights, without a GPU: every bad argument comes back as its status or a ValueError, and
nothing is launched."""
import ctypes

import pytest
import torch

from paper_2507_07145_amd import routing as r

NULL, BAD, UNSUPPORTED, ALIGN, WORKSPACE = -1, -2, -3, -4, -5
P = 4096   # a pointer that no call below may look behind


def order(**kw):
    return r.ccq_order(**{**dict(rows=P, experts=P, offsets=P, places=P), **kw})


def test_route():
    def call(o=None, ws=None, n=0, **kw):
        d = r.ccq_router(**{**dict(T=2, experts=64, top_k=8, groups=1, top_groups=1, group_best=1, scale=1.0, logits=P, ld=64, logits_type=1, ids=P, weights=P), **kw})
        return r._load().ccq_route(ctypes.byref(d), None if o is None else ctypes.byref(o), ws, n, None)
    assert r._load().ccq_route(None, None, None, 0, None) == NULL and r._load().ccq_route_workspace_bytes(None, 1) == -1
    assert call(T=0) == 0 and call(T=0, logits=None, ids=None) == 0
    for bad in (dict(T=-1), dict(experts=0), dict(top_k=0), dict(top_k=65), dict(scoring=2), dict(scoring=-1), dict(groups=0), dict(groups=7), dict(groups=8, top_groups=9),
                dict(groups=8, top_groups=0), dict(group_best=0), dict(group_best=3), dict(scale=float("nan")), dict(scale=float("inf")), dict(ld=63), dict(logits_type=2),
                dict(T=1 << 28, top_k=8)):
        assert call(**bad) == BAD, bad
    assert call(groups=16, top_groups=1) == BAD   # four experts are left, eight asked for
    assert call(experts=1025, ld=1025) == UNSUPPORTED and call(top_k=33) == UNSUPPORTED
    assert call(logits=None) == NULL and call(ids=None) == NULL and call(weights=None) == NULL
    assert call(logits=P + 2) == ALIGN and call(bias=P + 2) == ALIGN and call(ids=P + 2) == ALIGN and call(weights=P + 1) == ALIGN and call(logits=P + 1, logits_type=0) == ALIGN
    for o, status in ((order(rows=None), NULL), (order(offsets=None), NULL), (order(rows=P + 4), ALIGN), (order(offsets=P + 8), ALIGN), (order(places=P + 2), ALIGN), (order(experts=P + 1), ALIGN)):
        assert call(o) == status
    d = r.ccq_router(T=5000, experts=64, top_k=8, groups=1, top_groups=1, group_best=1, scale=1.0)
    need = r._load().ccq_route_workspace_bytes(ctypes.byref(d), 1)
    assert need > 0 and r._load().ccq_route_workspace_bytes(ctypes.byref(d), 0) == 0
    assert call(order(), T=5000) == WORKSPACE and call(order(), P, need - 1, T=5000) == WORKSPACE and call(order(), P + 4, need, T=5000) == ALIGN


def test_sort_rows():
    def call(o=None, ids=P, ld=3, T=2, k=3, first=0, experts=9, ws=None, n=0):
        o = order() if o is None else o
        return r._load().ccq_sort_rows(ids, ld, T, k, first, experts, ctypes.byref(o), ws, n, None)
    assert r._load().ccq_sort_rows(P, 3, 2, 3, 0, 9, None, None, 0, None) == NULL
    assert call(T=-1) == BAD and call(k=0) == BAD and call(experts=0) == BAD and call(first=-1) == BAD and call(ld=2) == BAD and call(T=1 << 30, k=2, ld=2) == BAD
    assert call(experts=4097) == UNSUPPORTED
    assert call(ids=None) == NULL and call(order(rows=None)) == NULL and call(order(offsets=None)) == NULL
    assert call(ids=P + 2) == ALIGN and call(order(rows=P + 4)) == ALIGN and call(order(offsets=P + 4)) == ALIGN
    size = r._load().ccq_sort_rows_workspace_bytes
    assert size(-1, 1, 1) == -1 and size(1, 0, 1) == -1 and size(1, 1, 4097) == -1 and size(0, 1, 1) == 0 and size(1 << 30, 1, 4096) > 0
    need = size(100000, 1, 64)
    assert need > 0 and call(T=100000, k=1, experts=64) == WORKSPACE and call(T=100000, k=1, experts=64, ws=P, n=need - 1) == WORKSPACE
    assert call(T=100000, k=1, experts=64, ws=P + 8, n=need) == ALIGN


def test_combine():
    def call(**kw):
        c = r.ccq_combination(**{**dict(T=2, k=3, N=64, P=6, rows=P, ld_rows=64, places=P, ld_places=3, weights=P, ld_weights=3, y=P, ldy=64), **kw})
        return r._load().ccq_combine(ctypes.byref(c), None)
    assert r._load().ccq_combine(None, None) == NULL and call(T=0) == 0 and call(T=0, rows=None, y=None) == 0
    for bad in (dict(T=-1), dict(k=0), dict(N=0), dict(P=-1), dict(ld_rows=63), dict(ld_places=2), dict(ld_weights=2), dict(ldy=63), dict(base=P + 64, ld_base=63), dict(base_type=2), dict(y_type=-1),
                dict(base=P, ld_base=128), dict(base=P, ld_base=64, base_type=1)):
        assert call(**bad) == BAD, bad
    assert call(rows=None) == NULL and call(places=None) == NULL and call(weights=None) == NULL and call(y=None) == NULL
    for off in (dict(rows=P + 1), dict(places=P + 2), dict(weights=P + 2), dict(y=P + 1), dict(y=P + 2, y_type=1), dict(base=P + 2, ld_base=64, base_type=1)):
        assert call(**off) == ALIGN, off


def test_adapters():
    def call(T=2, rows=P, experts=P, x=P, ldx=64, y=P, ldy=32, out=P, ld_out=32, ws=None, n=0, **kw):
        d = r.ccq_adapter_set(**{**dict(count=3, rank=16, K=64, N=32, a=P, b=P), **kw})
        return r._load().ccq_adapters(ctypes.byref(d), T, rows, experts, x, ldx, y, ldy, out, ld_out, ws, n, None)
    assert r._load().ccq_adapters(None, 1, P, P, P, 64, P, 32, P, 32, None, 0, None) == NULL and r._load().ccq_adapters_workspace_bytes(None, 1) == -1
    assert call(T=0) == 0 and call(T=0, x=None, out=None) == 0
    for bad in (dict(T=-1), dict(count=0), dict(rank=0), dict(K=0), dict(N=0), dict(ldx=63), dict(ldy=31), dict(ld_out=31), dict(ld_out=40), dict(K=(1 << 30) + 8, ldx=1 << 31)):
        assert call(**bad) == BAD, bad
    assert call(rank=264) == UNSUPPORTED and call(rank=12) == ALIGN and call(K=60) == ALIGN
    for null in (dict(a=None), dict(b=None), dict(rows=None), dict(experts=None), dict(x=None), dict(y=None), dict(out=None)):
        assert call(**null) == NULL, null
    for off in (dict(a=P + 8), dict(b=P + 8), dict(scales=P + 2), dict(ranks=P + 2), dict(rows=P + 2), dict(experts=P + 2), dict(x=P + 1), dict(y=P + 1), dict(out=P + 1), dict(ws=P + 4, n=1 << 20)):
        assert call(**off) == ALIGN, off
    d = r.ccq_adapter_set(count=3, rank=16, K=64, N=32)
    need = r._load().ccq_adapters_workspace_bytes(ctypes.byref(d), 2)
    assert need > 0 and call() == WORKSPACE and call(ws=P, n=need - 1) == WORKSPACE
    assert r._load().ccq_adapters_workspace_bytes(ctypes.byref(d), 0) == 0 and r._load().ccq_adapters_workspace_bytes(ctypes.byref(d), -1) == -1


def test_adapter_plans_fit_their_launches():
    """Workspaces of every size of call stay in proportion to it."""
    for count in (1, 7, 128, 4096):
        for rank in (8, 64, 256):
            for K, N in ((8, 1), (4096, 4096), (28672, 8192)):
                d = r.ccq_adapter_set(count=count, rank=rank, K=K, N=N)
                for T in (1, 2, 16, 17, 256, 257, 4096, 100000, 1 << 24):
                    need = r._load().ccq_adapters_workspace_bytes(ctypes.byref(d), T)
                    assert T * rank * 4 <= need <= 32 * T * (rank + 8) * 4, (count, rank, K, N, T)


def bf16(*s):
    return torch.zeros(s, dtype=torch.bfloat16)


def test_adapter_sets():
    with pytest.raises(ValueError, match="GPU"):
        r.Adapters(bf16(2, 8, 64), bf16(2, 32, 8))
    with pytest.raises(ValueError, match="contiguous"):
        r.Adapters(bf16(2, 64, 8).transpose(1, 2), bf16(2, 32, 8))
    with pytest.raises(ValueError, match="contiguous"):
        r.Adapters(bf16(2, 8, 64).float(), bf16(2, 32, 8).float())
    with pytest.raises(ValueError, match="beside"):
        r.Adapters(bf16(2, 8, 64), bf16(3, 32, 8))
    with pytest.raises(ValueError, match="scales"):
        r.Adapters(bf16(2, 8, 64), bf16(2, 32, 8), scales=torch.ones(3))
    with pytest.raises(ValueError, match="ranks"):
        r.Adapters(bf16(2, 8, 64), bf16(2, 32, 8), ranks=torch.ones(2))
    with pytest.raises(ValueError, match="nothing"):
        r.Adapters(bf16(0, 8, 64), bf16(0, 32, 8))


def test_host_tensors_and_wrong_types():
    for call in (lambda: r.route(torch.zeros(2, 8), 2), lambda: r.sort_rows(torch.zeros(2, 8, dtype=torch.int32), 2),
                 lambda: r.combine(bf16(4, 8), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2))):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="scoring"):
        r.route(torch.zeros(2, 8), 2, scoring="tanh")
    with pytest.raises(ValueError, match="logits"):
        r.route(torch.zeros(2, 8, dtype=torch.float16), 2)
    with pytest.raises(ValueError, match="bias"):
        r.route(torch.zeros(2, 8), 2, bias=torch.zeros(7))
    with pytest.raises(ValueError, match="ids"):
        r.sort_rows(torch.zeros(2, 8), 2)
    with pytest.raises(ValueError, match="weights"):
        r.combine(bf16(4, 8), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 3))
    with pytest.raises(ValueError, match="base"):
        r.combine(bf16(4, 8), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2), base=bf16(2, 9))
