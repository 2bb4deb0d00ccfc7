"""Rows that choose their weights: what stands around the grouped products of binding.py, and beside its shared ones.

    route        a router's logits to experts, weights and the order of rows that binding.grouped_gemm reads
    sort_rows    that order for ids that are there already: one GPU's share of the experts, the adapters of a batch's requests
    combine      the weighted sum of the experts' rows of each token
    adapters     low-rank adapters of many requests, beside a projection that all of them share

Argument marshalling only, as in layer.py (include/ccq.h says what each call computes): a native module (csrc/python/ccq_routing_call.cpp) takes the plain
cases with little host time, ctypes the others, which are checked and reported here.  Tensors are on the current GPU; with stream= the work is enqueued
there, and results that are made lie in that stream's memory.

The results of one call of route or sort_rows may be pieces of one allocation (of six tensors one, without stream=): who keeps one of them alone, or
saves it, takes a clone.

A layer of experts, without a copy to the host:

    routes = route(logits, 8, scoring="sigmoid", bias=balance, groups=8, top_groups=4, renormalize=True, scale=2.5)
    up = binding.grouped_gemm(w_up, x, routes.order.rows, routes.order.offsets)        # rows sorted by expert
    down = binding.grouped_gemm(w_down, activation(up), every_row, routes.order.offsets)      # every_row: 0, 1, 2 ...
    y = combine(down, routes.order.places, routes.weights, base=shared)
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from . import binding
from .binding import CcqError, _check, _stream_ptr, _t_ptr
from .layer import _answer, _f32, _gpu, _i32, _i64, _int32, _need, _on, _on_this_gpu, _own_rows, _rows, _type, _vp

_SCORING = {"softmax": 0, "sigmoid": 1}


class ccq_order(ctypes.Structure):
    _fields_ = [("rows", _vp), ("experts", _vp), ("offsets", _vp), ("places", _vp)]


class ccq_router(ctypes.Structure):
    _fields_ = [("T", _i32), ("experts", _i32), ("top_k", _i32), ("scoring", _i32), ("groups", _i32), ("top_groups", _i32), ("group_best", _i32), ("renormalize", _i32),
                ("scale", _f32), ("logits", _vp), ("ld", _i64), ("logits_type", _i32), ("bias", _vp), ("ids", _vp), ("weights", _vp)]


class ccq_combination(ctypes.Structure):
    _fields_ = [("T", _i32), ("k", _i32), ("N", _i32), ("P", _i32), ("rows", _vp), ("ld_rows", _i64), ("places", _vp), ("ld_places", _i64), ("weights", _vp), ("ld_weights", _i64),
                ("base", _vp), ("ld_base", _i64), ("base_type", _i32), ("y", _vp), ("ldy", _i64), ("y_type", _i32)]


class ccq_adapter_set(ctypes.Structure):
    _fields_ = [("count", _i32), ("rank", _i32), ("K", _i32), ("N", _i32), ("a", _vp), ("b", _vp), ("scales", _vp), ("ranks", _vp)]


_lib = None


def _load() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L, p = binding.load(), ctypes.POINTER
        for name, args in (("ccq_sort_rows", [_vp, _i64, _i32, _i32, _i32, _i32, p(ccq_order), _vp, _i64, _vp]), ("ccq_route", [p(ccq_router), p(ccq_order), _vp, _i64, _vp]),
                           ("ccq_combine", [p(ccq_combination), _vp]),
                           ("ccq_adapters", [p(ccq_adapter_set), _i32, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = ctypes.c_int, args
        for name, args in (("ccq_sort_rows_workspace_bytes", [_i32, _i32, _i32]), ("ccq_route_workspace_bytes", [p(ccq_router), _i32]),
                           ("ccq_adapters_workspace_bytes", [p(ccq_adapter_set), _i32])):
            f = getattr(L, name)
            f.restype, f.argtypes = _i64, args
        _lib = L
    return _lib


_native = None


def _calls():
    """The native module, given the library's entry points; raises if it has not been built."""
    global _native
    if _native is None:
        L = _load()
        try:
            from . import _ccq_routing as m
        except ImportError as e:
            raise RuntimeError("_ccq_routing.so is missing or does not load: build it with `python -m paper_2507_07145_amd.build`") from e
        m.bind(*(ctypes.cast(getattr(L, name), _vp).value for name in
                 ("ccq_route", "ccq_route_workspace_bytes", "ccq_sort_rows", "ccq_sort_rows_workspace_bytes", "ccq_combine", "ccq_adapters", "ccq_adapters_workspace_bytes")))
        _native = m
    return _native


class Order(NamedTuple):
    """Entries (t, j) sorted by expert, then t, then j, those of no expert after all others (int32): `rows` the t of each, `experts` its expert (-1: none), `offsets`
    [experts + 1] where each expert's begin, `places` [T][k] where each entry went (-1: no expert)."""
    rows: torch.Tensor
    experts: torch.Tensor
    offsets: torch.Tensor
    places: torch.Tensor


_new = tuple.__new__   # (past the Python code of a named tuple's own)


class Routes(NamedTuple):
    """ids int32 [T][k] (-1: none) and weights fp32 [T][k], the best expert first, and their order (None if it was not asked for)."""
    ids: torch.Tensor
    weights: torch.Tensor
    order: Order | None


class Adapters:
    """Low-rank adapters of one projection [N][K]: a bf16 [count][rank][K], b bf16 [count][N][rank], scales fp32 [count], ranks in use int32 [count]."""

    def __init__(self, a: torch.Tensor, b: torch.Tensor, scales: torch.Tensor | None = None, ranks: torch.Tensor | None = None):
        _need(a.dim() == 3 and b.dim() == 3 and a.dtype == b.dtype == torch.bfloat16 and a.is_contiguous() and b.is_contiguous(), "adapters: contiguous bf16 a [count][rank][K] and b [count][N][rank] are needed")
        count, rank, K = a.shape
        N = b.shape[1]
        _need(b.shape == (count, N, rank) and b.device == a.device, "adapters: b is [count][N][rank], beside a")
        for t, dtype, what in ((scales, torch.float32, "fp32 scales"), (ranks, torch.int32, "int32 ranks")):
            _need(t is None or (t.dtype == dtype and t.shape == (count,) and t.is_contiguous() and t.device == a.device), f"adapters: {what}, one per adapter, are needed")
        _int32(count, rank, K, N)
        _need(min(count, rank, K, N) > 0, "adapters: there is nothing in a or b")
        self.a, self.b, self.scales, self.ranks, self.gpu = a, b, scales, ranks, _gpu(a)
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self.desc = ccq_adapter_set(count, rank, K, N, a.data_ptr(), b.data_ptr(), ptr(scales), ptr(ranks))


def _ld(t: torch.Tensor) -> int:
    """Row stride; a single row's is whatever it is."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _new_order(T: int, k: int, experts: int, device) -> Order:
    new = lambda *shape: torch.empty(shape, dtype=torch.int32, device=device)  # noqa: E731
    return Order(new(T * k), new(T * k), new(experts + 1), new(T, k))


def _made_on(stream, make):
    """As layer._on, for several tensors at once."""
    made = []

    def one(i):
        if not made:
            made.extend(make())
        return made[i]
    out = [_on(stream, lambda: one(0))]
    return out + [_on(stream, lambda i=i: one(i)) for i in range(1, len(made))]


def _order_desc(o: Order) -> ccq_order:
    return ccq_order(*(t.data_ptr() for t in o))


def _workspace(need: int, stream, device, where: str):
    if need < 0:
        raise CcqError(-2, where)
    return _on(stream, lambda: binding._workspace(need, device), read_here=False)


def route(logits: torch.Tensor, top_k: int, scoring: str = "softmax", bias: torch.Tensor | None = None, groups: int = 1, top_groups: int | None = None, group_best: int = 2,
          renormalize: bool = False, scale: float = 1.0, order: bool = True, stream=None) -> Routes:
    """The top_k experts of each row of logits (bf16 or fp32 [T][experts]) by softmax or sigmoid scores plus bias (fp32 [experts], for the choice only), from the
    top_groups best of `groups` groups (all of them if not given), a group's value being the sum of its group_best largest; through ccq_route."""
    _need(scoring in _SCORING, f"scoring is one of {', '.join(_SCORING)}")
    if top_groups is None:
        top_groups = groups
    if stream is None:
        r = _answer((_native or _calls()).route(logits, top_k, _SCORING[scoring], bias, groups, top_groups, group_best, renormalize, float(scale), order), "ccq_route")
        if r is not None:
            return _new(Routes, (r[0], r[1], _new(Order, r[2:]) if order else None))
    _need(logits.dim() == 2 and logits.shape[1] > 0 and _rows(logits) and logits.dtype in (torch.bfloat16, torch.float32), "logits: bf16 or fp32 rows [T][experts] are needed")
    T, E = logits.shape
    _need(bias is None or (bias.shape == (E,) and bias.dtype == torch.float32 and (E == 1 or bias.stride(0) == 1)), "bias: fp32, one per expert, is needed")
    _on_this_gpu(logits, bias)
    _int32(T, E, top_k, groups, top_groups, group_best)
    r = ccq_router(T=T, experts=E, top_k=top_k, scoring=_SCORING[scoring], groups=groups, top_groups=top_groups, group_best=group_best, renormalize=bool(renormalize), scale=scale,
                   logits=logits.data_ptr(), ld=_ld(logits), logits_type=_type(logits), bias=None if bias is None else bias.data_ptr())
    L = _load()
    need = int(L.ccq_route_workspace_bytes(ctypes.byref(r), int(bool(order))))
    if need < 0:   # what is wrong, the call itself says
        _check(L.ccq_route(ctypes.byref(r), None, None, 0, _stream_ptr(stream)), "ccq_route")
    ids, weights = _made_on(stream, lambda: (torch.empty((T, top_k), dtype=torch.int32, device=logits.device), torch.empty((T, top_k), dtype=torch.float32, device=logits.device)))
    r.ids, r.weights = ids.data_ptr(), weights.data_ptr()
    sorted_ = Order(*_made_on(stream, lambda: _new_order(T, top_k, E, logits.device))) if order else None
    workspace = _workspace(need, stream, logits.device, "ccq_route")
    _check(L.ccq_route(ctypes.byref(r), ctypes.byref(_order_desc(sorted_)) if order else None, _t_ptr(workspace), 0 if workspace is None else workspace.nbytes, _stream_ptr(stream)),
           "ccq_route")
    return Routes(ids, weights, sorted_)


def sort_rows(ids: torch.Tensor, experts: int, first: int = 0, stream=None) -> Order:
    """The order of ids (int32 [T][k]) over the experts first .. first + experts - 1, through ccq_sort_rows; other ids are none."""
    if stream is None:
        r = _answer((_native or _calls()).sort(ids, experts, first), "ccq_sort_rows")
        if r is not None:
            return _new(Order, r)
    _need(ids.dim() == 2 and ids.dtype == torch.int32 and _rows(ids) and ids.shape[1] > 0, "ids: int32 rows [T][k] are needed")
    _on_this_gpu(ids)
    T, k = ids.shape
    _int32(T, k, experts, first)
    L = _load()
    need = int(L.ccq_sort_rows_workspace_bytes(T, k, experts))
    if need < 0:
        raise CcqError(-3 if experts > 4096 else -2, "ccq_sort_rows")
    o = Order(*_made_on(stream, lambda: _new_order(T, k, experts, ids.device)))
    workspace = _workspace(need, stream, ids.device, "ccq_sort_rows")
    _check(L.ccq_sort_rows(ids.data_ptr(), _ld(ids), T, k, first, experts, ctypes.byref(_order_desc(o)), _t_ptr(workspace), 0 if workspace is None else workspace.nbytes,
                           _stream_ptr(stream)), "ccq_sort_rows")
    return o


def combine(rows: torch.Tensor, places: torch.Tensor, weights: torch.Tensor, base: torch.Tensor | None = None, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """base[t] + sum over j of weights[t][j] rows[places[t][j]], through ccq_combine; bf16 rows, bf16 or fp32 base and out (bf16 if it is made)."""
    if stream is None:
        r = _answer((_native or _calls()).combine(rows, places, weights, base, out), "ccq_combine")
        if r is not None:
            return r
    _need(rows.dtype == torch.bfloat16 and _rows(rows), "rows: bf16 rows are needed")
    _need(places.dtype == torch.int32 and _rows(places) and places.shape[1:] != (0,), "places: int32 [T][k] are needed")
    T, N = places.shape[0], rows.shape[1]
    _need(weights.dtype == torch.float32 and weights.shape == places.shape and _rows(weights), "weights: fp32 like places are needed")
    _need(base is None or (base.shape == (T, N) and _rows(base)), "base: rows [T][N] are needed")
    _on_this_gpu(rows, places, weights, base, out)
    _int32(T, N, places.shape[1], rows.shape[0])
    if out is None:
        out = _on(stream, lambda: binding._new_output(T, N, rows.device))
    _need(out.shape == (T, N) and _rows(out) and _own_rows(out), "out: rows [T][N] of their own are needed")
    c = ccq_combination(T=T, k=places.shape[1], N=N, P=rows.shape[0], rows=rows.data_ptr(), ld_rows=_ld(rows), places=places.data_ptr(), ld_places=_ld(places),
                        weights=weights.data_ptr(), ld_weights=_ld(weights), y=out.data_ptr(), ldy=_ld(out), y_type=_type(out))
    if base is not None:
        c.base, c.ld_base, c.base_type = base.data_ptr(), _ld(base), _type(base)
    _check(_load().ccq_combine(ctypes.byref(c), _stream_ptr(stream)), "ccq_combine")
    return out


def adapters(y: torch.Tensor, x: torch.Tensor, adapters: Adapters, order: Order, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y + scale (x a^T) b^T with each row's adapter, through ccq_adapters; order: that of the rows' adapters (sort_rows of ids [T][1] over the adapters); out may be y."""
    if stream is None:
        r = _answer((_native or _calls()).adapters(y, x, adapters.desc, adapters.gpu, order.rows, order.experts, out, workspace), "ccq_adapters")
        if r is not None:
            return r
    d = adapters.desc
    _need(x.dtype == torch.bfloat16 and _rows(x) and x.shape[1] == d.K, "x: bf16 rows [T][K] are needed")
    T = x.shape[0]
    _need(y.dtype == torch.bfloat16 and _rows(y) and y.shape == (T, d.N), "y: bf16 rows [T][N] are needed")
    for t in (order.rows, order.experts):
        _need(t is not None and t.dtype == torch.int32 and t.shape == (T,) and (T <= 1 or t.stride(0) == 1), "order: one entry per row is needed")
    _on_this_gpu(x, y, adapters.a, order.rows, order.experts, out)
    _int32(T)
    if out is None:
        out = _on(stream, lambda: binding._new_output(T, d.N, x.device))
    _need(out.dtype == torch.bfloat16 and out.shape == (T, d.N) and _rows(out) and _own_rows(out), "out: bf16 rows [T][N] of their own are needed")
    if workspace is None:
        workspace = _workspace(adapters_workspace_bytes(adapters, T), stream, x.device, "ccq_adapters")
    else:
        binding._given_workspace(workspace, x)
    _check(_load().ccq_adapters(ctypes.byref(d), T, _t_ptr(order.rows), _t_ptr(order.experts), _t_ptr(x), _ld(x), _t_ptr(y), _ld(y), _t_ptr(out), _ld(out), _t_ptr(workspace),
                                0 if workspace is None else workspace.nbytes, _stream_ptr(stream)), "ccq_adapters")
    return out


def adapters_workspace_bytes(adapters: Adapters, T: int) -> int:
    _int32(T)
    need = int(_load().ccq_adapters_workspace_bytes(ctypes.byref(adapters.desc), T))
    if need < 0:   # what is wrong, the call itself says
        _check(_load().ccq_adapters(ctypes.byref(adapters.desc), T, None, None, None, adapters.desc.K, None, adapters.desc.N, None, adapters.desc.N, None, 0, None), "ccq_adapters")
        raise CcqError(-2, "ccq_adapters")
    return need
