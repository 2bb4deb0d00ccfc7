"""The operators of a decoder layer together, as the example has them: prompts against single tokens, and a replayed graph against eager steps."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

_spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "decoder_layer.py"))


@pytest.fixture(scope="module")
def example():
    m = importlib.util.module_from_spec(_spec)
    _spec.loader.exec_module(m)
    return m


def new(example, **sizes):
    torch.manual_seed(3)
    kind = dict(dict(layers=2, hidden=512, heads=8, kv_heads=2, feed_forward=1024, sequences=3, room=200), **sizes)
    return example.Decoder(**kind)


def test_a_prompt_and_its_tokens_one_by_one(example):
    """Both see the same tokens.  What differs: other kernels' order of sums and, in the cache, the rounding of a page whose scale rose later.  A rescaled value
    is rounded twice, 2^-4 of it each time at most; such errors are independent between tokens and dimensions, and the residual stream and the norm dampen
    them: the norm of the difference stays far below 2^-4 of the norm per layer, two layers here."""
    n, count = 37, 3
    decoder = new(example)
    x = torch.randn(count, n, 512, device="cuda").bfloat16()
    whole = decoder.prompt(x.view(count * n, 512)).view(count, n, 512).float()
    decoder.state.lens.zero_()
    single = torch.stack([decoder.token(x[:, t].contiguous()) for t in range(n)], 1).float()
    assert decoder.state.lens.tolist() == [n] * count
    assert torch.isfinite(whole).all()
    assert ((whole - single).norm() / whole.norm()).item() < 2 * 2.0**-4


def test_a_chunk_after_a_prompt(example):
    """The second chunk of a prompt gives what it gives in the whole prompt, by the argument above."""
    n, count = 150, 3
    decoder = new(example)
    x = torch.randn(count, n, 512, device="cuda").bfloat16()
    whole = decoder.prompt(x.view(count * n, 512)).view(count, n, 512).float()
    decoder.state.lens.zero_()
    parts = [decoder.prompt(x[:, a:b].reshape(-1, 512)).view(count, b - a, 512).float() for a, b in ((0, 70), (70, 71), (71, 150))]
    assert ((whole - torch.cat(parts, 1)).norm() / whole.norm()).item() < 2 * 2.0**-4


@pytest.mark.parametrize("sequences", [1, 3, 20])
def test_a_replayed_graph_gives_the_eager_steps(example, sequences):
    n, steps = 61, 8   # (the tokens pass the end of a page)
    decoder = new(example, sequences=sequences)
    prompt = torch.randn(sequences * n, 512, device="cuda").bfloat16()
    xs = torch.randn(steps, sequences, 512, device="cuda").bfloat16()

    def start():
        decoder.state.lens.zero_()
        decoder.prompt(prompt)

    start()
    eager = [decoder.token(x).clone() for x in xs]
    start()
    x = xs[0].clone()
    graph, y = example.capture(decoder, x)
    start()
    for i in range(steps):
        x.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), eager[i].view(torch.int16)), i
        torch.randn(1 << 16, device="cuda").sum().item()   # eager work of the program between replays
    assert decoder.state.lens.tolist() == [n + steps] * sequences
