"""Tensors behind the layer operators' descriptors that no kernel may be given.  Host only: nothing is launched."""
import ctypes
import threading

import pytest
import torch

from paper_2507_07145_amd import layer as l


def u8(*s):
    return torch.zeros(s, dtype=torch.uint8)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def test_rows_that_share_memory():
    """A kernel reads rows [i][width] of the table and of scales; of one row that was expanded to several there is only one."""
    with pytest.raises(ValueError, match="overlap"):
        l.Batch(i32(5), i32(4), i32(1, 3).expand(4, 3), 4, 1, 48)
    with pytest.raises(ValueError, match="overlap"):
        l.Batch(i32(5), i32(4), i32(6).as_strided((4, 3), (1, 1)), 4, 1, 48)
    with pytest.raises(ValueError, match="overlap"):
        l.Batch(i32(5), i32(4), i32(1, 1).expand(4, 1), 4, 1, 16)
    with pytest.raises(ValueError, match="overlap"):
        l.Weight8(u8(300, 256), torch.zeros(1, 2).expand(3, 2))
    for N in (128, 300):
        with pytest.raises(ValueError, match="overlap"):
            l.Rows8(u8(4, N), u8(1, -(-N // 128)).expand(4, -(-N // 128))).desc()


def test_tensors_on_the_host():
    """A descriptor holds addresses only, and kernels read there: its tensors have to lie on a GPU when it is made."""
    with pytest.raises(ValueError, match="GPU"):
        l.Weight8(u8(128, 256), torch.ones(1, 2))
    with pytest.raises(ValueError, match="GPU"):
        l.Cache8(u8(2, 1, 16, 64), u8(2, 1, 64, 16), u8(2, 1), u8(2, 1))
    with pytest.raises(ValueError, match="GPU"):
        l.Cache8.empty(2, 16, 1, 64, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        l.Batch(i32(3), i32(2), i32(2, 3), 2, 1, 3)
    with pytest.raises(ValueError, match="GPU"):
        l.Rope(torch.zeros(4, 8))


def test_workspaces_that_kernels_cannot_write():
    x = torch.empty(4, 128, device="meta")   # (another device than the workspaces')
    for ws, like in ((u8(64), x), (u8(64, 2)[:, 0], u8(1)), (u8(64, 2)[::2], u8(1))):
        with pytest.raises(ValueError, match="workspace"):
            l.binding._given_workspace(ws, like)
    ws = u8(64)
    assert l.binding._given_workspace(ws, u8(1)) is ws


def test_numbers_past_32_bits():
    """ctypes would cut them off: 2^32 + 5 tokens would be 5."""
    for kw in (dict(tokens=(1 << 32) + 2), dict(max_new=1 << 31), dict(max_len=(1 << 32) + 3), dict(max_len=-(1 << 31) - 1)):
        with pytest.raises(ValueError, match="31 bits"):
            l.Batch(i32(3), i32(2), i32(2, 3), **{**dict(tokens=2, max_new=1, max_len=48), **kw})
    with pytest.raises(ValueError, match="31 bits"):
        l.rope_table(1 << 32, 2, device="meta")
    with pytest.raises(ValueError, match="31 bits"):
        l.Rope(torch.empty((1 << 31, 2), device="meta"))
    with pytest.raises(ValueError, match="31 bits"):
        l.Weight8(torch.empty((1, 1 << 31), dtype=torch.uint8, device="meta"), torch.empty((1, 1 << 24), device="meta"))


def test_a_forced_kernel_is_the_threads_own():
    """The tests' switch does not reach the calls of other threads."""
    cache, batch = l.ccq_cache(64, 64, 8, 128, None, None, None, None), l.ccq_batch(1, 2048, 2048, 4096, None, None, None, 64, 64)
    need = lambda: l._load().ccq_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(l.ccq_attn(56, 1, 0, 1.0)))  # noqa: E731
    rule, other = need(), []
    l._load().ccq_attention_force(0)
    try:
        assert need() < rule
        t = threading.Thread(target=lambda: other.append(need()))
        t.start()
        t.join()
    finally:
        l._load().ccq_attention_force(-1)
    assert other == [rule]


def test_calls_past_what_a_launch_may_have():
    """2^32 threads and more are refused before the launch."""
    p = 4096   # a pointer that no call below may look behind
    cache = l.ccq_cache(4, 16, 2, 64, p, p, p, p)
    heads = l.ccq_heads(p, 256, 64)
    a = l.ccq_attn(4, 1, 0, 0.125)
    for tokens in (1 << 27, (1 << 26) + 64):
        batch = l.ccq_batch(2, tokens, tokens, 32, p, p, p, 2, 2)
        assert l._load().ccq_attention(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(a), ctypes.byref(heads), ctypes.byref(heads), None, 0, None) == -2
    w = l.ccq_weight8(128, 128, p, 128, p, 1)
    rows = l.ccq_rows8(p, 128, p, 1)
    for M in (0x7FFFFFFF, 0x7FFFFF01):
        assert l._load().ccq_gemm8(ctypes.byref(w), ctypes.byref(rows), M, p, 128, None, 0, None) == -2 and l._load().ccq_gemm8_workspace_bytes(ctypes.byref(w), M) == -1
        assert l._load().ccq_gemm8_bf16(ctypes.byref(w), p, 128, M, p, 128, p, 1 << 50, None) == -2 and l._load().ccq_gemm8_bf16_workspace_bytes(ctypes.byref(w), M) == -1
