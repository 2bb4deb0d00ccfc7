"""The layer operators' refusals, without a GPU: every bad argument comes back as its status, and nothing is launched."""
import ctypes

import pytest
import torch

from paper_2507_07145_amd import binding as b
from paper_2507_07145_amd import layer as l

NULL, BAD, UNSUPPORTED, ALIGN, WORKSPACE = -1, -2, -3, -4, -5
P = 4096   # a pointer that no call below may look behind


def ref(s):
    return None if s is None else ctypes.byref(s)


def norm(**kw):
    d = dict(M=2, N=128, eps=1e-6, x=P, ldx=128, y=P, ldy=128)
    d.update(kw)
    return l._load().ccq_rms_norm(ctypes.byref(l.ccq_norm(**d)), None)


def test_norm():
    r8 = lambda **kw: l.ccq_rows8(**{**dict(codes=P, ld=128, scales=P, ld_scales=1), **kw})  # noqa: E731
    assert l._load().ccq_rms_norm(None, None) == NULL
    assert norm(M=0) == 0 and norm(M=0, x=None) == 0
    assert norm(M=-1) == BAD and norm(N=0) == BAD and norm(eps=-1.0) == BAD and norm(eps=float("nan")) == BAD and norm(eps=float("inf")) == BAD
    assert norm(ldx=127) == BAD and norm(ldy=127) == BAD and norm(residual=P, ld_residual=5) == BAD and norm(residual=P, ld_residual=128, sum=P, ld_sum=1) == BAD
    assert norm(residual_type=2) == BAD and norm(weight=P, weight_type=-1) == BAD
    assert norm(residual=P, ld_residual=128, sum=P, ld_sum=256) == BAD and norm(y=P, ldx=256) == BAD   # on an input, but not row on row
    assert norm(x=None) == NULL and norm(y=None) == NULL
    assert norm(x=P + 1) == ALIGN and norm(residual=P + 2, ld_residual=128, residual_type=1) == ALIGN and norm(weight=P + 2, weight_type=1) == ALIGN
    assert norm(y8=r8(ld=127)) == BAD and norm(y8=r8(ld=120)) == BAD and norm(y8=r8(ld=136)) == ALIGN and norm(y8=r8(codes=P + 8)) == ALIGN and norm(y8=r8(scales=None)) == NULL
    assert norm(N=129, ldx=129, ldy=129, y8=r8(ld=144)) == BAD   # two blocks, one scale
    q = l._load().ccq_quantize8
    assert q(P, 128, 2, 128, None, None) == NULL and q(P, 128, 0, 128, ctypes.byref(r8()), None) == 0
    assert q(None, 128, 2, 128, ctypes.byref(r8()), None) == NULL and q(P, 100, 2, 128, ctypes.byref(r8()), None) == BAD and q(P, 128, 2, 128, ctypes.byref(r8(codes=None)), None) == NULL


def test_gemm8():
    def call(w={}, x={}, M=2, y=P, ldy=128, ws=None, n=0):
        wd = l.ccq_weight8(**{**dict(K=256, N=128, codes=P, ldw=256, scales=P, ld_scales=2), **w})
        xd = l.ccq_rows8(**{**dict(codes=P, ld=256, scales=P, ld_scales=2), **x})
        return l._load().ccq_gemm8(ctypes.byref(wd), ctypes.byref(xd), M, y, ldy, ws, n, None)
    assert l._load().ccq_gemm8(None, None, 1, None, 8, None, 0, None) == NULL
    assert call(M=0) == 0 and call(M=-1) == BAD
    assert call(w=dict(K=0)) == BAD and call(w=dict(N=0)) == BAD and call(w=dict(K=264, ldw=272, ld_scales=3)) == ALIGN and call(w=dict(ldw=240)) == BAD and call(w=dict(ldw=264)) == ALIGN
    assert call(w=dict(ld_scales=1)) == BAD and call(x=dict(ld=128)) == BAD and call(x=dict(ld=264)) == ALIGN and call(x=dict(ld_scales=1)) == BAD
    assert call(ldy=120) == BAD and call(ldy=129) == ALIGN and call(y=None) == NULL and call(w=dict(codes=None)) == NULL and call(w=dict(scales=None)) == NULL and call(x=dict(codes=None)) == NULL
    assert call(y=P + 8) == ALIGN and call(w=dict(codes=P + 8)) == ALIGN and call(x=dict(codes=P + 4)) == ALIGN and call(w=dict(scales=P + 4)) == ALIGN
    wd = l.ccq_weight8(28672, 512, P, 28672, P, 224)
    assert l._load().ccq_gemm8_workspace_bytes(None, 1) == -1 and l._load().ccq_gemm8_workspace_bytes(ctypes.byref(wd), -1) == -1
    needs = {M: l._load().ccq_gemm8_workspace_bytes(ctypes.byref(wd), M) for M in (0, 1, 16, 64, 200, 300, 2048)}
    assert needs[0] == 0 and all(n >= 0 for n in needs.values())
    for M, n in needs.items():
        if n:
            xd = l.ccq_rows8(P, 28672, P, 224)
            assert l._load().ccq_gemm8(ctypes.byref(wd), ctypes.byref(xd), M, P, 512, None, 0, None) == WORKSPACE
            assert l._load().ccq_gemm8(ctypes.byref(wd), ctypes.byref(xd), M, P, 512, P, n - 1, None) == WORKSPACE


def test_gemm8_of_bf16_rows():
    def call(w={}, x=P, ldx=256, M=2, y=P, ldy=128, ws=None, n=0):
        wd = l.ccq_weight8(**{**dict(K=256, N=128, codes=P, ldw=256, scales=P, ld_scales=2), **w})
        return l._load().ccq_gemm8_bf16(ctypes.byref(wd), x, ldx, M, y, ldy, ws, n, None)
    assert l._load().ccq_gemm8_bf16(None, P, 256, 1, P, 128, None, 0, None) == NULL
    assert call(M=0) == 0 and call(M=-1) == BAD and call(ldx=255) == BAD and call(x=None) == NULL and call(x=P + 1) == ALIGN and call(w=dict(K=0)) == BAD
    assert call(ldy=120) == BAD and call(ldy=129) == ALIGN and call(y=None) == NULL and call(w=dict(codes=None)) == NULL and call(y=P + 8) == ALIGN and call(ws=P + 8) == ALIGN
    wd = l.ccq_weight8(28672, 512, P, 28672, P, 224)
    need = l._load().ccq_gemm8_bf16_workspace_bytes
    assert need(None, 1) == -1 and need(ctypes.byref(wd), -1) == -1 and need(ctypes.byref(wd), 0) == 0
    n = need(ctypes.byref(wd), 2048)
    assert n >= 2048 * (28672 + 224)   # the 8-bit rows of a call that is served in blocks
    for ws, size in ((None, 0), (P, n - 1)):
        assert l._load().ccq_gemm8_bf16(ctypes.byref(wd), P, 28672, 2048, P, 512, ws, size, None) == WORKSPACE


def cache(**kw):
    return l.ccq_cache(**{**dict(pages=4, page_tokens=16, kv_heads=2, head_dim=64, k=P, v=P, k_scales=P, v_scales=P), **kw})


def batch(**kw):
    return l.ccq_batch(**{**dict(batch=2, tokens=2, max_new=1, max_len=32, offsets=P, lens=P, table=P, ld_table=2, table_width=2), **kw})


def heads(n, **kw):
    return l.ccq_heads(**{**dict(data=P, token_stride=64 * n, head_stride=64), **kw})


BAD_CACHES = [(dict(pages=0), BAD), (dict(kv_heads=0), BAD), (dict(page_tokens=0), BAD), (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED),
              (dict(page_tokens=512), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=0), BAD), (dict(k=None), NULL), (dict(v=None), NULL),
              (dict(k_scales=None), NULL), (dict(v_scales=None), NULL), (dict(k=P + 8), ALIGN), (dict(v=P + 8), ALIGN)]
BAD_BATCHES = [(dict(batch=-1), BAD), (dict(batch=70000), BAD), (dict(tokens=-1), BAD), (dict(max_new=-1), BAD), (dict(max_len=-1), BAD), (dict(max_len=(1 << 30) + 1), BAD),
               (dict(table_width=3), BAD), (dict(table_width=-1), BAD), (dict(offsets=None), NULL), (dict(lens=None), NULL), (dict(table=None), NULL), (dict(lens=P + 2), ALIGN)]


def append(c=None, ba=None, rope=None, k=2, v=2, q=4, o=4, q_heads=4):
    h = lambda n: heads(n) if type(n) is int else n  # noqa: E731
    c, ba = cache() if c is None else c, batch() if ba is None else ba
    return l._load().ccq_cache_append(ref(c), ref(ba), ref(rope), ref(h(k)), ref(h(v)), ref(h(q)), ref(h(o)), q_heads, None)


def test_append():
    for kw, status in BAD_CACHES:
        assert append(c=cache(**kw)) == status, kw
    for kw, status in BAD_BATCHES:
        assert append(ba=batch(**kw)) == status, kw
    for kw in (dict(batch=0), dict(tokens=0), dict(max_new=0)):
        assert append(ba=batch(**kw)) == 0
    assert append(k=None) == NULL and append(v=None) == NULL and append(q=None) == NULL and append(o=None) == NULL and append(k=None, v=None, q=None, o=None) == NULL
    assert append(q_heads=0) == BAD
    assert append(k=heads(2, data=None)) == NULL and append(k=heads(2, data=P + 8)) == ALIGN and append(v=heads(2, token_stride=132)) == ALIGN and append(v=heads(2, token_stride=120)) == BAD
    assert append(q=heads(4, head_stride=32)) == BAD and append(o=heads(4, head_stride=68, token_stride=512)) == ALIGN
    assert append(q=heads(4), o=heads(4, token_stride=512)) == BAD   # on the queries, but not row on row
    rope = lambda **kw: l.ccq_rope(**{**dict(table=P, rows=32, dims=64, interleaved=0, positions=None), **kw})  # noqa: E731
    for kw, status in ((dict(table=None), NULL), (dict(rows=0), BAD), (dict(dims=0), BAD), (dict(dims=63), BAD), (dict(dims=66), BAD), (dict(table=P + 2), ALIGN), (dict(positions=P + 1), ALIGN)):
        assert append(rope=rope(**kw)) == status, kw


def test_attention():
    def call(c=None, ba=None, q=None, o=None, ws=None, n=0, **kw):
        a = l.ccq_attn(**{**dict(q_heads=4, causal=1, window=0, scale=0.125), **kw})
        c, ba = cache() if c is None else c, batch() if ba is None else ba
        return l._load().ccq_attention(ctypes.byref(c), ctypes.byref(ba), ctypes.byref(a), ref(heads(4) if q is None else q), ref(heads(4) if o is None else o), ws, n, None)
    for kw, status in BAD_CACHES:
        assert call(c=cache(**kw)) == status, kw
    for kw, status in BAD_BATCHES:
        assert call(ba=batch(**kw)) == status, kw
    for kw in (dict(batch=0), dict(tokens=0), dict(max_new=0)):
        assert call(ba=batch(**kw)) == 0
    for kw in (dict(q_heads=0), dict(q_heads=3), dict(window=-1), dict(window=4, causal=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**kw) == BAD, kw
    assert call(ba=batch(tokens=1 << 30, max_new=1 << 30)) == BAD
    assert call(q=heads(4, data=None)) == NULL and call(o=heads(4, data=P + 2)) == ALIGN and call(q=heads(4, token_stride=260)) == ALIGN and call(o=heads(4, token_stride=192)) == BAD
    a = l.ccq_attn(4, 1, 0, 0.125)
    need = l._load().ccq_attention_workspace_bytes
    assert need(None, None, None) == -1 and need(ctypes.byref(cache(head_dim=96)), ctypes.byref(batch()), ctypes.byref(a)) == -1
    long = batch(batch=1, tokens=1, max_len=100000, table_width=6250, ld_table=6250)
    n = need(ctypes.byref(cache(pages=6250)), ctypes.byref(long), ctypes.byref(a))
    assert n > 0
    for ws, have in ((None, 0), (P, n - 1), (P + 4, n)):
        assert call(c=cache(pages=6250), ba=long, ws=ws, n=have) == (ALIGN if ws == P + 4 else WORKSPACE)


def test_rope_table():
    def call(rows=4, dims=8, table=P, **kw):
        s = l.ccq_rope_scaling(**{**dict(kind=0, base=10000.0, factor=2.0, original_length=4096.0, fast=32.0, slow=1.0, magnitude=1.0), **kw})
        return l._load().ccq_rope_table(ctypes.byref(s), rows, dims, table, None)
    assert l._load().ccq_rope_table(None, 1, 2, P, None) == NULL and call(table=None) == NULL and call(table=P + 2) == ALIGN and call(rows=0) == 0
    for kw in (dict(rows=-1), dict(dims=0), dict(dims=7), dict(kind=4), dict(kind=-1), dict(base=0.0), dict(base=float("inf")), dict(base=float("nan")), dict(magnitude=float("nan")),
               dict(kind=1, factor=0.0), dict(kind=1, factor=float("inf")), dict(kind=2, dims=2), dict(kind=3, original_length=0.0), dict(kind=3, fast=0.5), dict(kind=3, slow=0.0),
               dict(kind=3, base=1.0)):
        assert call(**kw) == BAD, kw


def test_python_refusals():
    """What the Python side says of tensors that do not fit, before any entry point is called."""
    u8, f32, i32 = (lambda *s: torch.zeros(s, dtype=torch.uint8)), (lambda *s: torch.zeros(s)), (lambda *s: torch.zeros(s, dtype=torch.int32))  # noqa: E731
    for codes, scales in ((f32(4, 128), f32(1, 1)), (u8(4, 128), f32(1, 2)), (u8(4, 128), u8(1, 1)), (u8(128, 4).t(), f32(1, 1))):
        with pytest.raises(ValueError):
            l.Weight8(codes, scales)
    with pytest.raises(ValueError):
        l.Rows8(u8(4, 129), u8(4, 1)).desc()
    for k, v, s in ((u8(2, 1, 16, 64), u8(2, 1, 16, 64), u8(2, 1)), (u8(2, 1, 16, 64), u8(2, 1, 64, 16), u8(2, 2)), (f32(2, 1, 16, 64), f32(2, 1, 64, 16), u8(2, 1))):
        with pytest.raises(ValueError):
            l.Cache8(k, v, s, s)
    for offsets, lens, table in ((i32(2), i32(2), i32(2, 3)), (i32(3), i32(2), i32(3, 3)), (f32(3), i32(2), i32(2, 3))):
        with pytest.raises(ValueError):
            l.Batch(offsets, lens, table, 2, 1, 3)
    with pytest.raises(ValueError):
        l.Rope(f32(4, 8), dims=6)
    with pytest.raises(ValueError):
        l.rope_table(4, 8, kind="other")
    for x in (torch.zeros(2, 128), torch.zeros(2, 128, dtype=torch.bfloat16)):   # fp32; not on a GPU
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            l.rms_norm(x, None)
    assert b.load() is l._load()
