"""The rest of a decoder layer, in 8 bits: the operators between the quantized products of binding.py.

    rms_norm      residual, root-mean-square norm, bf16 rows (for binding.gemm) or 8-bit rows (for gemm8)
    quantize8     bf16 rows as 8-bit rows
    gemm8         product with 8-bit weights, one scale per block of 128 x 128
    rope_table    cosines and sines of rotary positions
    cache_append  rotary positions, new keys and values into a paged 8-bit cache
    attention     over that cache: single new tokens or chunks of prompts

Argument marshalling only, as in binding.py (include/ccq.h says what each call computes): a native module
(csrc/python/ccq_layer_call.cpp) takes the plain cases with little host time, ctypes the others, which are checked and reported here.

Weight8, Cache8, Batch and Rope hold tensors of one GPU, and calls are made with that GPU current.  With stream= the work is enqueued there; results that are
made lie in that stream's memory, and the current stream has to wait for it before it reads them.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import CcqError, _check, _stream_ptr, _t_ptr

BLOCK = 128     # columns per scale of 8-bit rows and weights
BF16, FP32 = 0, 1

_vp, _i32, _i64, _f32, _f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double


class ccq_rows8(ctypes.Structure):
    _fields_ = [("codes", _vp), ("ld", _i64), ("scales", _vp), ("ld_scales", _i64)]


class ccq_norm(ctypes.Structure):
    _fields_ = [("M", _i32), ("N", _i32), ("eps", _f32), ("x", _vp), ("ldx", _i64), ("residual", _vp), ("ld_residual", _i64), ("sum", _vp), ("ld_sum", _i64),
                ("residual_type", _i32), ("weight", _vp), ("weight_type", _i32), ("y", _vp), ("ldy", _i64), ("y8", ccq_rows8)]


class ccq_weight8(ctypes.Structure):
    _fields_ = [("K", _i32), ("N", _i32), ("codes", _vp), ("ldw", _i64), ("scales", _vp), ("ld_scales", _i64)]


class ccq_cache(ctypes.Structure):
    _fields_ = [("pages", _i32), ("page_tokens", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("k", _vp), ("v", _vp), ("k_scales", _vp), ("v_scales", _vp)]


class ccq_batch(ctypes.Structure):
    _fields_ = [("batch", _i32), ("tokens", _i32), ("max_new", _i32), ("max_len", _i32), ("offsets", _vp), ("lens", _vp), ("table", _vp),
                ("ld_table", _i64), ("table_width", _i32)]


class ccq_heads(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class ccq_rope(ctypes.Structure):
    _fields_ = [("table", _vp), ("rows", _i32), ("dims", _i32), ("interleaved", _i32), ("positions", _vp)]


class ccq_rope_scaling(ctypes.Structure):
    _fields_ = [("kind", _i32), ("base", _f64), ("factor", _f64), ("original_length", _f64), ("fast", _f64), ("slow", _f64), ("magnitude", _f64)]


class ccq_attn(ctypes.Structure):
    _fields_ = [("q_heads", _i32), ("causal", _i32), ("window", _i32), ("scale", _f32)]


_lib = None


def _load() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L, p = binding.load(), ctypes.POINTER
        for name, args in (("ccq_rms_norm", [p(ccq_norm), _vp]), ("ccq_quantize8", [_vp, _i64, _i32, _i32, p(ccq_rows8), _vp]),
                           ("ccq_gemm8", [p(ccq_weight8), p(ccq_rows8), _i32, _vp, _i64, _vp, _i64, _vp]),
                           ("ccq_gemm8_bf16", [p(ccq_weight8), _vp, _i64, _i32, _vp, _i64, _vp, _i64, _vp]),
                           ("ccq_rope_table", [p(ccq_rope_scaling), _i32, _i32, _vp, _vp]),
                           ("ccq_cache_append", [p(ccq_cache), p(ccq_batch), p(ccq_rope), p(ccq_heads), p(ccq_heads), p(ccq_heads), p(ccq_heads), _i32, _vp]),
                           ("ccq_attention", [p(ccq_cache), p(ccq_batch), p(ccq_attn), p(ccq_heads), p(ccq_heads), _vp, _i64, _vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = ctypes.c_int, args
        for f in (L.ccq_gemm8_workspace_bytes, L.ccq_gemm8_bf16_workspace_bytes):
            f.restype, f.argtypes = _i64, [p(ccq_weight8), _i32]
        L.ccq_attention_workspace_bytes.restype, L.ccq_attention_workspace_bytes.argtypes = _i64, [p(ccq_cache), p(ccq_batch), p(ccq_attn)]
        _lib = L
    return _lib


_native = None


def _calls():
    """The native module, given the library's entry points; raises if it has not been built."""
    global _native
    if _native is None:
        L = _load()
        try:
            from . import _ccq_layer as m
        except ImportError as e:
            raise RuntimeError("_ccq_layer.so is missing or does not load: build it with `python -m paper_2507_07145_amd.build`") from e
        m.bind(*(ctypes.cast(getattr(L, name), _vp).value for name in
                 ("ccq_rms_norm", "ccq_quantize8", "ccq_gemm8", "ccq_gemm8_workspace_bytes", "ccq_cache_append", "ccq_attention", "ccq_attention_workspace_bytes",
                  "ccq_gemm8_bf16", "ccq_gemm8_bf16_workspace_bytes")))
        _native = m
    return _native


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _int32(*values: int) -> None:
    """The entry points take these numbers in 32 bits, and ctypes cuts off what does not fit."""
    for v in values:
        _need(-(1 << 31) <= v < 1 << 31, "sizes and counts of up to 31 bits are needed")


def _on_this_gpu(*tensors) -> None:
    for t in tensors:
        if t is not None:
            _need(t.is_cuda and t.device.index == torch.cuda.current_device(), "tensors have to be on the current GPU")


def _gpu(t) -> int:
    """The GPU whose memory a descriptor points to: kernels read what lies behind it unseen."""
    _need(t.is_cuda, "tensors on a GPU are needed")
    return t.device.index


def _is_codes(t) -> bool:
    return t.dtype in (torch.uint8, torch.float8_e4m3fn)


def _is_scales(t) -> bool:
    return t.dtype in (torch.uint8, torch.float8_e8m0fnu)


def _rows(t) -> bool:
    return t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1)


def _ld(t) -> int:
    """Row stride; a single row's is whatever it is."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), (t.shape[1] + 15) // 16 * 16)


def _own_rows(t) -> bool:
    """Rows that do not share memory, as rows made by expand do."""
    return t.shape[0] <= 1 or t.stride(0) >= t.shape[1]


def _type(t) -> int:
    _need(t.dtype in (torch.bfloat16, torch.float32), "bf16 or fp32 is needed")
    return FP32 if t.dtype == torch.float32 else BF16


class Rows8:
    """Rows of e4m3 values with a power-of-two scale (a byte e + 127) per row and block of 128 columns."""
    __slots__ = ("codes", "scales")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        self.codes, self.scales = codes, scales

    @property
    def shape(self):
        return self.codes.shape

    def desc(self) -> ccq_rows8:
        c, s = self.codes, self.scales
        _need(_is_codes(c) and _rows(c) and _is_scales(s) and _rows(s), "8-bit rows: codes [M][N] and scales [M][ceil(N / 128)] are needed")
        _need(s.shape == (c.shape[0], -(-c.shape[1] // BLOCK)) and s.device == c.device, "8-bit rows: one scale per row and block of 128 columns is needed")
        _need(_own_rows(s), "8-bit rows: rows of scales must not overlap")
        return ccq_rows8(c.data_ptr(), _ld(c), s.data_ptr(), max(s.stride(0), s.shape[1]))


def _on(stream, make, read_here: bool = True):
    """What `make` allocates for work on `stream` (None: the current one), from that stream's memory: the current stream's may still be in use there by
    kernels whose tensors were dropped.  A result is kept until the current stream has read it."""
    if stream is None:
        return make()
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        t = make()
    for x in (t.codes, t.scales) if type(t) is Rows8 else (t,) if read_here and t is not None else ():
        x.record_stream(here)
    return t


def _new_rows8(M: int, N: int, device) -> Rows8:
    codes = torch.empty((M, (N + 15) // 16 * 16), dtype=torch.uint8, device=device)[:, :N]
    return Rows8(codes, torch.empty((M, -(-N // BLOCK)), dtype=torch.uint8, device=device))


class Weight8:
    """8-bit weights [N][K] (e4m3) with one fp32 scale per block of 128 x 128."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        _need(_is_codes(codes) and _rows(codes), "8-bit weights: codes [N][K] are needed")
        N, K = codes.shape
        _need(scales.dtype == torch.float32 and _rows(scales) and scales.shape == (-(-N // BLOCK), -(-K // BLOCK)) and scales.device == codes.device,
              "8-bit weights: fp32 scales [ceil(N / 128)][ceil(K / 128)] are needed")
        _need(_own_rows(scales), "8-bit weights: rows of scales must not overlap")
        _int32(N, K)
        self.codes, self.scales, self.gpu = codes, scales, _gpu(codes)
        self.desc = ccq_weight8(K, N, codes.data_ptr(), _ld(codes), scales.data_ptr(), max(scales.stride(0), scales.shape[1]))

    @property
    def K(self):
        return self.desc.K

    @property
    def N(self):
        return self.desc.N


class Cache8:
    """A paged cache of e4m3 keys [pages][heads][page tokens][dim] and values [pages][heads][dim][page tokens], scales [pages][heads]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor):
        _need(k.dim() == 4 and _is_codes(k) and _is_codes(v) and k.is_contiguous() and v.is_contiguous(), "cache: contiguous 8-bit keys and values are needed")
        pages, heads, page_tokens, dim = k.shape
        _need(v.shape == (pages, heads, dim, page_tokens), "cache: values are [pages][heads][dim][page tokens]")
        for s in (k_scales, v_scales):
            _need(_is_scales(s) and s.is_contiguous() and s.shape == (pages, heads), "cache: scales are contiguous bytes [pages][heads]")
        _need(k.device == v.device == k_scales.device == v_scales.device, "cache: all on one device")
        _int32(pages)
        self.k, self.v, self.k_scales, self.v_scales, self.gpu = k, v, k_scales, v_scales, _gpu(k)
        self.desc = ccq_cache(pages, page_tokens, heads, dim, k.data_ptr(), v.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr())

    @classmethod
    def empty(cls, pages: int, page_tokens: int, kv_heads: int, head_dim: int, device="cuda") -> "Cache8":
        """A cache with nothing in it (its memory is not cleared: slots that are not written are never looked at)."""
        new = lambda *shape: torch.empty(shape, dtype=torch.uint8, device=device)  # noqa: E731
        return cls(new(pages, kv_heads, page_tokens, head_dim), new(pages, kv_heads, head_dim, page_tokens), new(pages, kv_heads), new(pages, kv_heads))


class Batch:
    """The sequences of a step: offsets [B + 1] of their new token rows, lengths [B] with the new tokens, page table [B][width] (int32, on
    the GPU); `tokens` token rows, at most `max_new` new tokens and `max_len` tokens in a sequence.  A loop that keeps its
    tensors and updates them in place keeps the object; max_len may then be what the table holds."""

    def __init__(self, offsets: torch.Tensor, lens: torch.Tensor, table: torch.Tensor, tokens: int, max_new: int, max_len: int):
        for t in (offsets, lens, table):
            _need(t.dtype == torch.int32 and t.device == offsets.device, "batch: int32 tensors on one device are needed")
        B = lens.shape[0]
        _need(lens.dim() == 1 and (B <= 1 or lens.stride(0) == 1) and offsets.shape == (B + 1,) and (B == 0 or offsets.stride(0) == 1),
              "batch: offsets [B + 1] and lens [B] are needed")
        _need(_rows(table) and table.shape[0] == B, "batch: a table [B][pages of a sequence] is needed")
        _need(_own_rows(table), "batch: rows of the table must not overlap")
        _int32(B, tokens, max_new, max_len, table.shape[1])
        self.offsets, self.lens, self.table, self.gpu = offsets, lens, table, _gpu(lens)
        self.desc = ccq_batch(B, tokens, max_new, max_len, offsets.data_ptr(), lens.data_ptr(), table.data_ptr(), max(table.stride(0), table.shape[1]), table.shape[1])


class Rope:
    """Rotary positions: table [positions][dims] fp32 (cosines, then sines), pairs (i, i + dims / 2) or, interleaved, (2 i, 2 i + 1)."""

    def __init__(self, table: torch.Tensor, dims: int | None = None, interleaved: bool = False, positions: torch.Tensor | None = None):
        dims = table.shape[1] if dims is None else dims
        _need(table.dtype == torch.float32 and table.is_contiguous() and table.dim() == 2 and table.shape[1] == dims, "rope: a contiguous fp32 table [positions][dims] is needed")
        _need(positions is None or (positions.dtype == torch.int32 and positions.is_contiguous() and positions.dim() == 1 and positions.device == table.device),
              "rope: int32 positions, one per token row, are needed")
        _int32(table.shape[0], dims)
        self.table, self.positions, self.gpu = table, positions, _gpu(table)
        self.desc = ccq_rope(table.data_ptr(), table.shape[0], dims, int(interleaved), None if positions is None else positions.data_ptr())


_KINDS = {"none": 0, "linear": 1, "base": 2, "parts": 3}


def rope_table(rows: int, dims: int, base: float = 10000.0, kind: str = "none", factor: float = 1.0, original_length: float = 0.0, fast: float = 32.0,
               slow: float = 1.0, magnitude: float = 1.0, device="cuda", stream=None) -> torch.Tensor:
    """Cosines and sines of positions 0 .. rows - 1, fp32 [rows][dims], through ccq_rope_table; `kind` is the scaling for contexts longer
    than the trained one: "none", "linear", "base" or "parts"."""
    _need(kind in _KINDS, f"kind is one of {', '.join(_KINDS)}")
    _int32(rows, dims)
    out = _on(stream, lambda: torch.empty((rows, dims), dtype=torch.float32, device=device))
    s = ccq_rope_scaling(_KINDS[kind], base, factor, original_length, fast, slow, magnitude)
    with torch.cuda.device(out.device):
        _check(_load().ccq_rope_table(ctypes.byref(s), rows, dims, _t_ptr(out), _stream_ptr(stream)), "ccq_rope_table")
    return out


def _answer(r, where: str):
    if type(r) is int:
        _check(r, where)
        return None
    return r


def rms_norm(x: torch.Tensor, weight: torch.Tensor | None, eps: float = 1e-6, residual: torch.Tensor | None = None, residual_out: torch.Tensor | None = None,
             out: torch.Tensor | None = None, rows8: bool = False, stream=None):
    """Norm of x (+ residual): bf16 rows, or Rows8 with `rows8` (with `out` too, both are written).  The sum goes to `residual_out`, or to `residual`
    itself."""
    if stream is None:
        r = _answer((_native or _calls()).rms_norm(x, weight, float(eps), residual, residual_out, out, rows8), "ccq_rms_norm")
        if r is not None:
            return Rows8(*r) if rows8 else r
    _need(x.dtype == torch.bfloat16 and _rows(x) and x.shape[1] > 0, "x: bf16 rows are needed")
    _on_this_gpu(x, weight, residual, residual_out, out)
    M, N = x.shape
    _int32(M, N)
    n = ccq_norm(M=M, N=N, eps=eps, x=x.data_ptr(), ldx=_ld(x))
    if weight is not None:
        _need(weight.shape == (N,) and (N == 1 or weight.stride(0) == 1), "weight: one per column is needed")
        n.weight, n.weight_type = weight.data_ptr(), _type(weight)
    _need(residual is not None or residual_out is None, "residual_out needs a residual")
    if residual is not None:
        total = residual if residual_out is None else residual_out
        _need(residual.shape == x.shape and _rows(residual) and total.shape == x.shape and _rows(total) and total.dtype == residual.dtype,
              "residual and residual_out: rows like x's, of one type, are needed")
        n.residual, n.ld_residual, n.residual_type = residual.data_ptr(), _ld(residual), _type(residual)
        n.sum, n.ld_sum = total.data_ptr(), _ld(total)
    y8 = _on(stream, lambda: _new_rows8(M, N, x.device)) if rows8 else None
    if rows8:
        n.y8 = y8.desc()
    elif out is None:
        out = _on(stream, lambda: binding._new_output(M, N, x.device))
    if out is not None:
        _need(out.dtype == torch.bfloat16 and out.shape == x.shape and _rows(out), "out: bf16 rows like x's are needed")
        n.y, n.ldy = out.data_ptr(), _ld(out)
    _check(_load().ccq_rms_norm(ctypes.byref(n), _stream_ptr(stream)), "ccq_rms_norm")
    return y8 if rows8 else out


def quantize8(x: torch.Tensor, stream=None) -> Rows8:
    """bf16 rows as 8-bit rows, through ccq_quantize8."""
    if stream is None:
        r = _answer((_native or _calls()).quantize8(x), "ccq_quantize8")
        if r is not None:
            return Rows8(*r)
    _need(x.dtype == torch.bfloat16 and _rows(x) and x.shape[1] > 0, "x: bf16 rows are needed")
    _on_this_gpu(x)
    _int32(*x.shape)
    out = _on(stream, lambda: _new_rows8(*x.shape, x.device))
    d = out.desc()
    _check(_load().ccq_quantize8(_t_ptr(x), _ld(x), x.shape[0], x.shape[1], ctypes.byref(d), _stream_ptr(stream)), "ccq_quantize8")
    return out


def gemm8(w: Weight8, x, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = x W^T through ccq_gemm8; x: Rows8, or bf16 rows, whose 8-bit rows are formed on the way (ccq_gemm8_bf16)."""
    is8 = type(x) is Rows8
    if stream is None:
        r = _answer((_native or _calls()).gemm8(w.desc, w.gpu, x.codes if is8 else x, x.scales if is8 else None, out, workspace), "ccq_gemm8")
        if r is not None:
            return r
    _need(is8 or (x.dtype == torch.bfloat16 and _rows(x)), "x: Rows8 or bf16 rows are needed")
    held = x.codes if is8 else x
    _on_this_gpu(held, w.codes, out)
    M, N = x.shape[0], w.N
    _int32(M)
    _need(x.shape[1] == w.K, "x and the weights have another K")
    y = _on(stream, lambda: binding._new_output(M, N, held.device)) if out is None else out
    _need(y.dtype == torch.bfloat16 and y.shape == (M, N) and _rows(y), "out: bf16 rows [M][N] are needed")
    if workspace is None:
        workspace = _on(stream, lambda: binding._workspace(gemm8_workspace_bytes(w, M, not is8), y.device), read_here=False)
    else:
        binding._given_workspace(workspace, held)
    tail = (M, _t_ptr(y), y.stride(0) if M > 1 else (N + 7) // 8 * 8, _t_ptr(workspace), 0 if workspace is None else workspace.nbytes, _stream_ptr(stream))
    if is8:
        _check(_load().ccq_gemm8(ctypes.byref(w.desc), ctypes.byref(x.desc()), *tail), "ccq_gemm8")
    else:
        _check(_load().ccq_gemm8_bf16(ctypes.byref(w.desc), _t_ptr(x), _ld(x), *tail), "ccq_gemm8_bf16")
    return y


def gemm8_workspace_bytes(w: Weight8, M: int, bf16_rows: bool = False) -> int:
    _int32(M)
    f = _load().ccq_gemm8_bf16_workspace_bytes if bf16_rows else _load().ccq_gemm8_workspace_bytes
    need = int(f(ctypes.byref(w.desc), M))
    if need < 0:
        raise CcqError(-2, f.__name__)
    return need


def _heads(t: torch.Tensor, tokens: int, heads: int | None, dim: int, name: str) -> ccq_heads:
    _need(t.dim() == 3 and t.dtype == torch.bfloat16 and t.shape[0] == tokens and t.shape[2] == dim and t.stride(2) == 1 and (heads is None or t.shape[1] == heads),
          f"{name}: bf16 [tokens][heads][head dim], the last side by side, is needed")
    head = t.stride(1) if t.shape[1] > 1 else dim
    return ccq_heads(t.data_ptr(), t.stride(0) if tokens > 1 else max(t.stride(0), (t.shape[1] - 1) * head + dim), head)


def cache_append(cache: Cache8, batch: Batch, k: torch.Tensor | None, v: torch.Tensor | None, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
                 rope: Rope | None = None, stream=None) -> torch.Tensor | None:
    """New keys (rotated) and values into the cache, and q rotated (returned; None without q), through ccq_cache_append."""
    if rope is not None and rope.positions is not None:
        _need(rope.positions.numel() >= batch.desc.tokens, "rope: a position per token row is needed")
    if stream is None:
        r = (_native or _calls()).append(cache.desc, cache.gpu, batch.desc, batch.gpu, k, v, q, q_out, None if rope is None else rope.desc, cache.gpu if rope is None else rope.gpu)
        if type(r) is int:
            _check(r, "ccq_cache_append")
            return None
        if r is not None:
            return r
    _on_this_gpu(cache.k, batch.lens, k, v, q, q_out, None if rope is None else rope.table)
    T, H, D = batch.desc.tokens, cache.desc.kv_heads, cache.desc.head_dim
    hk, hv = (None if t is None else _heads(t, T, H, D, n) for t, n in ((k, "k"), (v, "v")))
    hq = ho = None
    if q is not None:
        hq = _heads(q, T, None, D, "q")
        q_out = _on(stream, lambda: torch.empty(q.shape, dtype=q.dtype, device=q.device)) if q_out is None else q_out
        ho = _heads(q_out, T, q.shape[1], D, "q_out")
    else:
        _need(q_out is None, "q_out needs a q")
    ref = lambda s: None if s is None else ctypes.byref(s)  # noqa: E731
    _check(_load().ccq_cache_append(ctypes.byref(cache.desc), ctypes.byref(batch.desc), ref(None if rope is None else rope.desc), ref(hk), ref(hv), ref(hq), ref(ho),
                                    0 if q is None else q.shape[1], _stream_ptr(stream)), "ccq_cache_append")
    return q_out


def attention(cache: Cache8, batch: Batch, q: torch.Tensor, scale: float | None = None, window: int = 0, causal: bool = True, out: torch.Tensor | None = None,
              workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """softmax(scale q k^T) v over the cache, through ccq_attention; scale: 1 / sqrt(head dim) if not given."""
    if scale is None:
        scale = cache.desc.head_dim ** -0.5
    if stream is None:
        r = _answer((_native or _calls()).attention(cache.desc, cache.gpu, batch.desc, batch.gpu, q, float(scale), window, causal, out, workspace), "ccq_attention")
        if r is not None:
            return r
    _on_this_gpu(cache.k, batch.lens, q, out)
    T, D = batch.desc.tokens, cache.desc.head_dim
    hq = _heads(q, T, None, D, "q")
    out = _on(stream, lambda: torch.empty(q.shape, dtype=q.dtype, device=q.device)) if out is None else out
    ho = _heads(out, T, q.shape[1], D, "out")
    _int32(window, q.shape[1])
    a = ccq_attn(q.shape[1], int(bool(causal)), window, scale)
    if workspace is None:
        need = int(_load().ccq_attention_workspace_bytes(ctypes.byref(cache.desc), ctypes.byref(batch.desc), ctypes.byref(a)))
        if need < 0:
            raise CcqError(-2, "ccq_attention")
        workspace = _on(stream, lambda: binding._workspace(need, q.device), read_here=False)
    else:
        binding._given_workspace(workspace, q)
    _check(_load().ccq_attention(ctypes.byref(cache.desc), ctypes.byref(batch.desc), ctypes.byref(a), ctypes.byref(hq), ctypes.byref(ho), _t_ptr(workspace),
                                 0 if workspace is None else workspace.nbytes, _stream_ptr(stream)), "ccq_attention")
    return out
