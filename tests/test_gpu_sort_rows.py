"""The order of rows by expert: a permutation with its offsets and places, exactly."""
import numpy as np
import pytest
import torch

from paper_2507_07145_amd import routing
from test_gpu_route import check_order

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ids_of(T, k, lo, hi, seed):
    return torch.randint(lo, hi, (T, k), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)


@pytest.mark.parametrize("T,k", [(1, 1), (1, 8), (63, 1), (64, 1), (65, 1), (100, 3), (1023, 1), (1024, 1), (1025, 1), (2047, 1), (2048, 1), (2049, 1), (700, 6), (5000, 2), (16384, 8), (140000, 1)])
@pytest.mark.parametrize("experts", [1, 2, 63, 64, 256, 1000, 4096])
def test_sizes(T, k, experts):
    ids = ids_of(T, k, 0, experts, T + experts)
    check_order(routing.sort_rows(ids.to(DEV), experts), ids.numpy(), experts, f"{T} x {k} over {experts}")


def test_ids_of_no_expert():
    ids = ids_of(3000, 4, -3, 80, 1)
    ids[5] = torch.tensor([-2 ** 31, 2 ** 31 - 1, -1, 64])
    for first, experts in ((0, 64), (0, 80), (16, 16), (79, 1), (2 ** 31 - 1, 8), (70, 4096)):
        check_order(routing.sort_rows(ids.to(DEV), experts, first=first), ids.numpy(), experts, f"{first}, {experts}", first=first)
    none = torch.full((200, 2), -1, dtype=torch.int32)
    check_order(routing.sort_rows(none.to(DEV), 7), none.numpy(), 7, "none at all")
    one = torch.full((9000, 1), 5, dtype=torch.int32)
    check_order(routing.sort_rows(one.to(DEV), 7), one.numpy(), 7, "all of one")


def test_no_rows():
    o = routing.sort_rows(torch.empty(0, 3, dtype=torch.int32, device=DEV), 5)
    assert o.offsets.tolist() == [0] * 6 and o.places.shape == (0, 3)


def test_strides_and_stream():
    wide = ids_of(500, 11, 0, 32, 2).to(DEV)
    for view in (wide[:, 2:5], wide[::3, :1], wide[7:8, 1:9]):
        check_order(routing.sort_rows(view, 32), view.cpu().numpy(), 32, "view")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    o = routing.sort_rows(wide, 32, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    check_order(o, wide.cpu().numpy(), 32, "stream")


@pytest.mark.parametrize("T,k", [(40, 8), (6000, 2)])
def test_captured(T, k):
    ids = ids_of(T, k, 0, 64, 3).to(DEV)
    routing.sort_rows(ids, 64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = routing.sort_rows(ids, 64)
    for seed in (4, 5, 6):
        ids.copy_(ids_of(T, k, -1, 70, seed))
        graph.replay()
        check_order(o, ids.cpu().numpy(), 64, "replay")
        check_order(routing.sort_rows(ids, 64), ids.cpu().numpy(), 64, "eager")


def test_behind_the_arrays():
    """Nothing is written past the arrays' ends."""
    import ctypes
    ids = ids_of(70, 3, -1, 9, 7).to(DEV)
    room = [torch.full((n + 8,), -7, dtype=torch.int32, device=DEV) for n in (210, 210, 10, 210)]
    o = routing.ccq_order(*(t.data_ptr() for t in room))
    assert routing._load().ccq_sort_rows(ids.data_ptr(), 3, 70, 3, 0, 9, ctypes.byref(o), None, 0, None) == 0
    torch.cuda.synchronize()
    for t, n in zip(room, (210, 210, 10, 210)):
        assert np.all(t[n:].cpu().numpy() == -7)
    o = routing.ccq_order(room[0].data_ptr(), None, room[2].data_ptr(), None)   # (experts and places are optional)
    assert routing._load().ccq_sort_rows(ids.data_ptr(), 3, 70, 3, 0, 9, ctypes.byref(o), None, 0, None) == 0
    check_order(routing.Order(room[0][:210], room[1][:210], room[2][:10], room[3][:210].view(70, 3)), ids.cpu().numpy(), 9, "without experts and places")


@pytest.mark.parametrize("T,k,experts", [(4096, 1, 7), (4097, 1, 7), (1024, 2, 1), (8192, 1, 3), (8193, 1, 30), (2731, 3, 4096), (512, 8, 1024), (8192, 1, 300), (131072, 8, 9), (65536, 8, 1024), (262144, 8, 256), (300001, 7, 4096)])
def test_many_workgroups(T, k, experts):
    ids = ids_of(T, k, -1, experts, T)
    check_order(routing.sort_rows(ids.to(DEV), experts), ids.numpy(), experts, f"{T} x {k} over {experts}")
