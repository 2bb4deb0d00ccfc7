"""Decoder layers of a language model on one GPU: attention in 8 bits, the feed-forward part in CCQ's 2 bits.

    python examples/decoder_layer.py [--layers 2 --hidden 4096 --heads 32 --kv-heads 8 --feed-forward 8192 --prompt 512 --sequences 4 --steps 32]

Weights are random.  A prompt goes through the layers at once, then tokens one by one: eagerly, and as a captured graph that is replayed.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2507_07145_amd import binding as ccq  # noqa: E402
from paper_2507_07145_amd import layer  # noqa: E402

PAGE_TOKENS = 64


def weight8(W: torch.Tensor) -> layer.Weight8:
    """fp32 [N][K] as e4m3 with a scale per block of 128 x 128."""
    N, K = W.shape
    nb, kb = -(-N // layer.BLOCK), -(-K // layer.BLOCK)
    blocks = torch.zeros((nb * layer.BLOCK, kb * layer.BLOCK), device=W.device)
    blocks[:N, :K] = W
    scales = (blocks.view(nb, layer.BLOCK, kb, layer.BLOCK).abs().amax((1, 3)) / 448).clamp_min(1e-30)
    codes = blocks / scales.repeat_interleave(layer.BLOCK, 0).repeat_interleave(layer.BLOCK, 1)
    return layer.Weight8(codes[:N, :K].contiguous().to(torch.float8_e4m3fn), scales)


class Sequences:
    """Page table and lengths of a batch of sequences, each with room for `room` tokens."""

    def __init__(self, sequences: int, room: int, device="cuda"):
        self.count, width = sequences, -(-room // PAGE_TOKENS)
        self.pages, self.room = sequences * width, width * PAGE_TOKENS
        self.table = torch.arange(self.pages, dtype=torch.int32, device=device).view(sequences, width)
        self.lens = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.one_each = self.step(1)

    def step(self, n: int) -> layer.Batch:
        """A step of n new tokens in every sequence; lens has to count them when it runs."""
        offsets = torch.arange(0, n * self.count + 1, n, dtype=torch.int32, device=self.lens.device)
        return layer.Batch(offsets, self.lens, self.table, n * self.count, n, self.room)


class DecoderLayer:
    def __init__(self, hidden: int, heads: int, kv_heads: int, feed_forward: int, pages: int, rope: layer.Rope, head_dim: int = 128, device="cuda"):
        new = lambda n, k: torch.randn(n, k, device=device) * k**-0.5  # noqa: E731
        self.heads, self.kv_heads, self.head_dim, self.feed_forward, self.rope = heads, kv_heads, head_dim, feed_forward, rope
        self.norm_in, self.norm_mid = torch.ones(hidden, device=device), torch.ones(hidden, device=device)
        self.qkv = weight8(new((heads + 2 * kv_heads) * head_dim, hidden))
        self.o = weight8(new(hidden, heads * head_dim))
        self.gate_up = ccq.quantize(new(2 * feed_forward, hidden), ccq.NARROW)
        self.down = ccq.quantize(new(hidden, feed_forward), ccq.NARROW)
        self.cache = layer.Cache8.empty(pages, PAGE_TOKENS, kv_heads, head_dim, device)

    def __call__(self, x: torch.Tensor, stream_sum: torch.Tensor, batch: layer.Batch) -> torch.Tensor:
        """Adds x to the residual stream (fp32, in place) and returns what the layer adds to it next."""
        T, H, G, D = x.shape[0], self.heads, self.kv_heads, self.head_dim
        rows = layer.rms_norm(x, self.norm_in, residual=stream_sum, rows8=True)
        qkv = layer.gemm8(self.qkv, rows).view(T, H + 2 * G, D)
        q = layer.cache_append(self.cache, batch, qkv[:, H : H + G], qkv[:, H + G :], qkv[:, :H], rope=self.rope)
        attended = layer.attention(self.cache, batch, q)
        o = layer.gemm8(self.o, attended.view(T, H * D))
        y = ccq.gemm(self.gate_up, layer.rms_norm(o, self.norm_mid, residual=stream_sum))
        act = torch.nn.functional.silu(y[:, : self.feed_forward]) * y[:, self.feed_forward :]
        return ccq.gemm(self.down, act)


class Decoder:
    def __init__(self, layers: int, hidden: int, heads: int, kv_heads: int, feed_forward: int, sequences: int, room: int, device="cuda"):
        self.state = Sequences(sequences, room, device)
        rope = layer.Rope(layer.rope_table(self.state.room, 128, device=device))
        self.layers = [DecoderLayer(hidden, heads, kv_heads, feed_forward, self.state.pages, rope, device=device) for _ in range(layers)]
        self.norm_out = torch.ones(hidden, device=device)

    def __call__(self, x: torch.Tensor, batch: layer.Batch) -> torch.Tensor:
        """bf16 [tokens][hidden] through the layers, normed."""
        total = torch.zeros(x.shape, device=x.device)
        for one in self.layers:
            x = one(x, total, batch)
        return layer.rms_norm(x, self.norm_out, residual=total)

    def prompt(self, x: torch.Tensor) -> torch.Tensor:
        """n tokens of every sequence, after what is cached: bf16 [sequences n][hidden]."""
        n = x.shape[0] // self.state.count
        self.state.lens += n
        return self(x, self.state.step(n))

    def token(self, x: torch.Tensor) -> torch.Tensor:
        """One token of every sequence; its tensors are the same in every step, so that a graph may hold it."""
        self.state.lens += 1
        return self(x, self.state.one_each)


def capture(decoder: Decoder, x: torch.Tensor):
    """The step of one token as a graph that reads x and counts the cached tokens up; returns it and the tensor that it writes."""
    before = decoder.state.lens.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):   # once outside, then for the graph
        decoder.token(x)
    torch.cuda.current_stream().wait_stream(side)
    decoder.state.lens.copy_(before)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = decoder.token(x)
    return graph, y


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("layers", 2), ("hidden", 4096), ("heads", 32), ("kv-heads", 8), ("feed-forward", 8192), ("prompt", 512), ("sequences", 4), ("steps", 32)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args()
    torch.manual_seed(0)
    decoder = Decoder(a.layers, a.hidden, a.heads, a.kv_heads, a.feed_forward, a.sequences, a.prompt + 3 * a.steps)
    x = torch.randn(a.sequences * a.prompt, a.hidden, device="cuda").bfloat16()
    decoder.prompt(x)
    decoder.state.lens.zero_()

    def timed(what, run, times):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(times):
            run()
        torch.cuda.synchronize()
        print(f"{what}: {(time.perf_counter() - t) / times * 1e6:.1f} us", flush=True)

    timed(f"{a.sequences} prompts of {a.prompt}", lambda: decoder.prompt(x), 1)
    step = x[: a.sequences].clone()
    timed(f"a token of {a.sequences} sequences, eager", lambda: decoder.token(step), a.steps)
    graph, _ = capture(decoder, step)
    timed(f"a token of {a.sequences} sequences, graph", graph.replay, a.steps)


if __name__ == "__main__":
    main()
