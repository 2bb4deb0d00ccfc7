"""The native host path of routing.py's functions (_ccq_routing.so) behaves as the general Python path does around the launch."""
import ctypes

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2507_07145_amd import routing

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Calls:
    """One call of each function, as the native module takes it and as a program makes it."""

    def __init__(self):
        g = torch.Generator(DEV).manual_seed(1)
        bf16 = lambda *s: torch.randn(s, device=DEV, generator=g).bfloat16()  # noqa: E731
        self.logits, self.bias = torch.randn(30, 24, device=DEV, generator=g), torch.zeros(24, device=DEV)
        self.ids = torch.arange(40, dtype=torch.int32, device=DEV)[:, None] % 5 - 1
        self.order = routing.sort_rows(self.ids, 4)
        self.rows, self.places, self.weights = bf16(60, 72), torch.arange(60, dtype=torch.int32, device=DEV).view(30, 2), torch.rand(30, 2, device=DEV, generator=g)
        self.adapters, self.x, self.y = routing.Adapters(bf16(4, 8, 64), bf16(4, 72, 8)), bf16(40, 64), bf16(40, 72)
        self.out30, self.out40 = torch.empty(30, 72, dtype=torch.bfloat16, device=DEV), torch.empty(40, 72, dtype=torch.bfloat16, device=DEV)
        self.workspace = torch.empty(routing.adapters_workspace_bytes(self.adapters, 40), dtype=torch.uint8, device=DEV)

    def native(self, m, logits=None, ids=None, rows=None, x=None):
        pick = lambda a, b: b if a is None else a  # noqa: E731
        a = self.adapters
        return (m.route(pick(logits, self.logits), 4, 0, self.bias, 4, 2, 2, True, 1.0, True), m.sort(pick(ids, self.ids), 4, 0),
                m.combine(pick(rows, self.rows), self.places, self.weights, None, self.out30),
                m.adapters(self.y, pick(x, self.x), a.desc, a.gpu, self.order.rows, self.order.experts, self.out40, self.workspace))

    def made(self, like=lambda t: t):
        r = routing.route(like(self.logits), 4, bias=self.bias, groups=4, top_groups=2, renormalize=True)
        return [r.ids, r.weights, *r.order, *routing.sort_rows(like(self.ids), 4), routing.combine(like(self.rows), self.places, self.weights),
                routing.adapters(self.y, like(self.x), self.adapters, self.order)]


def test_other_threads_run_during_a_call(monkeypatch):
    """The entry points run without the interpreter lock.  CPython's own PyGILState_Check stands in for those that launch (nothing is launched): it returns 0, which is CCQ_OK,
    only where the calling thread does not hold the lock."""
    c = Calls()
    check = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    real = lambda name: ctypes.cast(getattr(routing._load(), name), ctypes.c_void_p).value  # noqa: E731
    m = routing._calls()
    monkeypatch.setattr(routing, "_native", None)            # (the next call binds the library's entry points again)
    m.bind(check, real("ccq_route_workspace_bytes"), check, real("ccq_sort_rows_workspace_bytes"), check, check, real("ccq_adapters_workspace_bytes"))
    try:
        route, order, combined, adapted = c.native(m)
    finally:
        routing._calls()
    assert len(route) == 6 and len(order) == 4 and combined is c.out30 and adapted is c.out40


class _Record(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.seen = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.seen.append(str(func))
        return func(*args, **(kwargs or {}))


def test_a_dispatch_mode_sees_what_is_allocated():
    """Memory trackers and tensor wrappers work by a TorchDispatchMode: results and workspaces come through it."""
    c = Calls()
    want = c.made()
    with _Record() as r:
        got = c.made()
    assert sum(s.startswith("aten.empty") for s in r.seen) == len(want) + 1, r.seen      # (and the adapters' workspace)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_subclass_is_not_looked_into():
    c = Calls()
    sub = lambda t: t.as_subclass(type("Sub", (torch.Tensor,), {}))  # noqa: E731
    assert c.native(routing._calls(), sub(c.logits), sub(c.ids), sub(c.rows), sub(c.x)) == (None,) * 4
    assert all(torch.equal(a, b) for a, b in zip(c.made(sub), c.made()))


def test_out_of_memory_is_the_allocators_exception():
    """A result that does not fit raises torch.OutOfMemoryError, as torch.empty does (the limit is the allocator's own, set from here: nothing is launched).
    On a stream of their own: what earlier work has left free in pieces of the current one's memory is not for it."""
    T = 1 << 23
    logits, ids = torch.zeros(T, 8, dtype=torch.bfloat16, device=DEV), torch.zeros(T, 8, dtype=torch.int32, device=DEV)
    weights, rows = torch.zeros(T, 8, device=DEV), torch.zeros(1, 64, dtype=torch.bfloat16, device=DEV)
    a = routing.Adapters(torch.zeros(1, 8, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(1, 64, 8, dtype=torch.bfloat16, device=DEV))
    x = torch.zeros(T, 64, dtype=torch.bfloat16, device=DEV)
    order = routing.Order(ids[:, 0].contiguous(), ids[:, 0].contiguous(), None, None)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    torch.cuda.set_per_process_memory_fraction(0.0)
    try:
        for call in (lambda: routing.route(logits, 8), lambda: routing.sort_rows(ids, 4), lambda: routing.combine(rows, ids, weights), lambda: routing.adapters(x, x, a, order)):
            with torch.cuda.stream(stream), pytest.raises(torch.OutOfMemoryError):
                call()
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert routing.route(logits[:4], 2).ids.shape == (4, 2)
