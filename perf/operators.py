"""The operators that stand between the quantized products of a decoder layer, as a serving program calls them.

Four kinds of case, through the public functions of `paper_2507_07145_amd.layer`:

  norm       h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight, as bf16 rows (what `binding.gemm` reads) or as e4m3 rows
             with one power-of-two scale per row and block of 128 columns (what `layer.gemm8` reads).
  gemm8      y = x W^T on e4m3 weights with one fp32 scale per block of 128 x 128: the layers of a model that stay at 8 bits.
             `x` says what the program has in hand: "rows8" the 8-bit rows of a norm, "bf16" rows that the call quantizes.
  append     rotary positions on q and k (fp32 table of cosines and sines), k and v of new tokens written to a paged cache of
             e4m3 values with one power-of-two scale per page and head.  A page that holds tokens already keeps its scale or
             takes a larger one, to which its older tokens are brought.
  attention  softmax(scale q k^T) v over that cache, B sequences of ragged lengths: one new token each (decode) or a chunk of a
             prompt, causal, with or without a sliding window.

Scales with a power of two are bytes e + 127 that stand for 2^e.  Slots of a page that no token was written to hold NaN.
"""
import math
import random

import torch

own = False

BLOCK = 128            # columns per scale
E4M3_MAX = 448.0
EPS = 1e-6
CACHE_EXP = 60         # exponents of the cache's scales lie in [-60, 60]

# the largest of each kind: what draw() stays below
MAX_NORM = 2048 * 18432
MAX_GEMM = 2048 * 7168 * 18432
MAX_KN = 28672 * 8192
MAX_TOKENS = 4096
MAX_PAIRS = 56 * 2048 * 4096
MAX_CACHED = 64 * 8192 * 8 * 128


def listed():
    return [
        # one token's hidden state between two layers: launch and call overhead
        {"name": "norm-1x8192", "kind": "norm", "M": 1, "N": 8192, "residual": True, "out": "bf16"},
        # a prefill chunk, rows for the 8-bit projections
        {"name": "norm-2048x7168", "kind": "norm", "M": 2048, "N": 7168, "residual": True, "out": "rows8"},
        # one token through a square projection
        {"name": "gemm8-1x8192", "kind": "gemm8", "M": 1, "K": 8192, "N": 8192, "x": "rows8"},
        # a decode batch through an output projection, from the attention's bf16 rows, ragged in every dimension
        {"name": "gemm8-37x7184", "kind": "gemm8", "M": 37, "K": 7184, "N": 5001, "x": "bf16"},
        # a prefill chunk through an up projection
        {"name": "gemm8-2048x18432", "kind": "gemm8", "M": 2048, "K": 7168, "N": 18432, "x": "rows8"},
        # a decode batch's new tokens: 64 query heads, 8 key heads, whole head rotated
        {"name": "append-decode-64", "kind": "append", "B": 64, "n": 1, "kv": 8192, "Hq": 64, "Hkv": 8, "D": 128, "P": 64, "rot": 128, "pairs": "half"},
        # a prompt of 2048 tokens on 1000 cached ones, part of the head rotated, neighbouring pairs
        {"name": "append-prompt-2048", "kind": "append", "B": 1, "n": 2048, "kv": 3048, "Hq": 56, "Hkv": 8, "D": 128, "P": 64, "rot": 64, "pairs": "neighbours"},
        # the smallest: four short conversations on a small model
        {"name": "attn-short-4", "kind": "attention", "B": 4, "n": 1, "kv": 200, "Hq": 16, "Hkv": 4, "D": 64, "P": 16, "window": 0},
        # one long conversation
        {"name": "attn-long-1", "kind": "attention", "B": 1, "n": 1, "kv": 131072, "Hq": 64, "Hkv": 8, "D": 128, "P": 64, "window": 0},
        # a decode batch of ragged lengths
        {"name": "attn-decode-64", "kind": "attention", "B": 64, "n": 1, "kv": 8192, "Hq": 32, "Hkv": 8, "D": 128, "P": 64, "window": 0},
        # a prefill chunk on as many cached tokens
        {"name": "attn-prompt-2048", "kind": "attention", "B": 1, "n": 2048, "kv": 4096, "Hq": 56, "Hkv": 8, "D": 128, "P": 64, "window": 0},
        # chunks of several prompts at once, sliding window, odd lengths
        {"name": "attn-window-6", "kind": "attention", "B": 6, "n": 301, "kv": 2999, "Hq": 32, "Hkv": 8, "D": 128, "P": 32, "window": 1024},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "gemm8", "gemm8", "append", "attention", "attention", "attention"])
    while True:
        if kind == "norm":
            case = {"M": _log(rng, 1, 4096), "N": _log(rng, 256, 18432), "residual": rng.random() < 0.75, "out": rng.choice(("bf16", "rows8"))}
            if rng.random() < 0.5:
                case["N"] = case["N"] // 64 * 64
            fits = case["M"] * case["N"] <= MAX_NORM
        elif kind == "gemm8":
            case = {"M": _log(rng, 1, 2048), "K": 16 * _log(rng, 16, 1792), "N": _log(rng, 500, 28672), "x": rng.choice(("rows8", "bf16"))}
            if rng.random() < 0.5:
                case["K"], case["N"] = (case["K"] + 127) // 128 * 128, (case["N"] + 63) // 64 * 64
            fits = case["M"] * case["K"] * case["N"] <= MAX_GEMM and case["K"] * case["N"] <= MAX_KN
        else:
            n = rng.choice((1, _log(rng, 2, 16), _log(rng, 16, 2048)))
            D = rng.choice((64, 128, 128))
            case = {"B": _log(rng, 1, 128), "n": n, "kv": max(n, _log(rng, 64, 65536)), "Hkv": rng.choice((1, 2, 4, 8)), "D": D, "P": rng.choice((16, 32, 64, 128))}
            case["Hq"] = case["Hkv"] * rng.choice((1, 2, 4, 5, 7, 8))
            lengths = _lengths(case)
            fits = sum(lengths[0]) <= MAX_TOKENS and case["B"] * case["kv"] * case["Hkv"] * D <= MAX_CACHED
            if kind == "append":
                case["rot"], case["pairs"] = rng.choice((D, D, D // 2)), rng.choice(("half", "neighbours"))
            else:
                case["window"] = rng.choice((0, 0, _log(rng, 32, 4096)))
                fits = fits and case["B"] * case["n"] * case["Hq"] * case["kv"] <= MAX_PAIRS
        if fits:
            return {"kind": kind, **case}


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 16 + stream) & (2 ** 62 - 1))


def _normal(shape, seed, stream, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=_gen(seed, stream))


def _hidden(M, N, seed, stream):
    """Hidden states: normal, a few columns much larger than the others, as trained models have them."""
    x = _normal((M, N), seed, stream)
    x[:, :: max(1, N // 5)] *= 20.0
    return x.to(torch.bfloat16)


def _lengths(case):
    """(new tokens, length with them) of each sequence: the first has the most of both."""
    r = random.Random(case["B"] * 1000003 + case["kv"] * 101 + case["n"])
    n = [case["n"]] + [r.randint(max(1, case["n"] // 4), case["n"]) for _ in range(case["B"] - 1)]
    kv = [case["kv"]] + [max(m, int(case["kv"] * r.uniform(0.25, 1.0))) for m in n[1:]]
    return n, kv


def _pow2(byte):
    """2^(byte - 127) in fp32."""
    return torch.exp2(byte.float() - 127.0)


def _exponent(amax, lo, hi):
    """The least e in [lo, hi] with amax <= 448 * 2^e, as a byte e + 127."""
    m, x = torch.frexp(amax)                     # amax = m 2^x, m in [0.5, 1); 448 = 0.875 * 2^9
    e = x - 9 + (m > 0.875).to(x.dtype)
    e = torch.where(amax > 0, e, torch.full_like(e, lo))
    return (e.clamp(lo, hi) + 127).to(torch.uint8)


def _prepare_batch(case, seed):
    n, kv = _lengths(case)
    B, P = case["B"], case["P"]
    need = [(k + P - 1) // P for k in kv]
    total, width = sum(need) + 3, max(need)
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed) & (2 ** 62 - 1)))
    table, at = torch.full((B, width), -1, dtype=torch.int32), 0
    for i, c in enumerate(need):
        table[i, :c] = order[at:at + c].to(torch.int32)
        at += c
    offsets = torch.tensor([0] + n, dtype=torch.int32).cumsum(0).to(torch.int32)
    return {"table": table.cuda(), "offsets": offsets.cuda(), "kv": torch.tensor(kv, dtype=torch.int32).cuda(), "pages": total,
            "T": sum(n), "n": n, "lens": kv}


def _prepare_cache(case, seed, b, written):
    """Pages of e4m3 values with their scales; `written[i]` tokens of sequence i are there, the other slots hold NaN."""
    shape = (b["pages"], case["Hkv"], case["P"], case["D"])
    out = []
    for stream in (4, 5):
        v = _normal(shape, seed, stream)
        if stream == 4:
            v[..., :: case["D"] // 4] *= 4.0     # keys: a few large channels
        v *= torch.exp2(_normal((b["pages"], case["Hkv"], 1, 1), seed, stream + 2))
        byte = _exponent(v.abs().amax((2, 3)), -CACHE_EXP, CACHE_EXP)
        codes = (v / _pow2(byte)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        del v
        filled = torch.zeros(b["pages"], dtype=torch.int64, device="cuda")
        first = torch.arange(b["table"].shape[1], device="cuda") * case["P"]
        count = (torch.tensor(written, device="cuda")[:, None] - first).clamp(0, case["P"])
        have = b["table"] >= 0
        filled[b["table"][have].long()] = count[have]
        empty = torch.arange(case["P"], device="cuda") >= filled[:, None]
        codes.masked_fill_(empty[:, None, :, None], 0x7F)
        out += [codes if stream == 4 else codes.transpose(2, 3).contiguous(), byte]
    return dict(zip(("k", "k_scales", "v", "v_scales"), out))


def _rope_table(rows, rot, base=10000.0):
    """Cosines, then sines, of the angles of each position: fp32 [rows][rot]."""
    freq = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    angle = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat((angle.cos(), angle.sin()), 1).float()


def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case}
    if kind == "norm":
        s["x"] = _hidden(case["M"], case["N"], seed, 0)
        s["weight"] = (1.0 + _normal((case["N"],), seed, 1, 0.1)).to(torch.bfloat16)
        if case["residual"]:
            s["residual"] = _hidden(case["M"], case["N"], seed, 2)
            s["sum"] = torch.empty_like(s["residual"])
    elif kind == "gemm8":
        M, K, N = case["M"], case["K"], case["N"]
        kb, nb = -(-K // BLOCK), -(-N // BLOCK)
        w = torch.zeros((nb * BLOCK, kb * BLOCK), device="cuda")
        w[:N, :K].normal_(0.0, 0.02, generator=_gen(seed, 0))
        blocks = w.view(nb, BLOCK, kb, BLOCK)
        s["w_scales"] = blocks.abs().amax((1, 3)) / E4M3_MAX
        s["w"] = (blocks / s["w_scales"][:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(nb * BLOCK, kb * BLOCK)[:N, :K].contiguous()
        del w, blocks
        x = _hidden(M, K, seed, 1)
        if case["x"] == "rows8":
            s["x8"], s["x_scales"] = _rows8(x.float())
        else:
            s["x"] = x
    else:
        b = s["batch"] = _prepare_batch(case, seed)
        held = [k - (n if kind == "append" else 0) for n, k in zip(b["n"], b["lens"])]
        s["cache"] = _prepare_cache(case, seed, b, held)
        s["q"] = _normal((b["T"], case["Hq"], case["D"]), seed, 0).to(torch.bfloat16)
        if kind == "append":
            s["k"] = (3.0 * _normal((b["T"], case["Hkv"], case["D"]), seed, 1)).to(torch.bfloat16)
            s["v"] = _normal((b["T"], case["Hkv"], case["D"]), seed, 2).to(torch.bfloat16)
            s["rope"] = _rope_table(case["kv"], case["rot"])
    if own:   # the handles that a program makes once and keeps
        from paper_2507_07145_amd import layer
        if kind == "gemm8":
            s["own_w"] = layer.Weight8(s["w"], s["w_scales"])
            if case["x"] == "rows8":
                s["own_x"] = layer.Rows8(s["x8"], s["x_scales"])
        elif kind != "norm":
            c, b = s["cache"], s["batch"]
            s["own_cache"] = layer.Cache8(c["k"], c["v"], c["k_scales"], c["v_scales"])
            s["own_batch"] = layer.Batch(b["offsets"], b["kv"], b["table"], tokens=b["T"], max_new=case["n"], max_len=case["kv"])
            if kind == "append":
                s["own_rope"] = layer.Rope(s["rope"], case["rot"], interleaved=case["pairs"] == "neighbours")
    return s


# ---- the plain forms: 32 bits, rounded once ---------------------------------------------------------------------------

def _rows8(y):
    """fp32 rows as e4m3 values and bytes of scales, one per row and block of BLOCK columns."""
    M, N = y.shape
    nb = -(-N // BLOCK)
    blocks = torch.zeros((M, nb * BLOCK), device=y.device)
    blocks[:, :N] = y
    blocks = blocks.view(M, nb, BLOCK)
    byte = _exponent(blocks.abs().amax(2), -126, 120)
    codes = (blocks / _pow2(byte)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8).view(M, nb * BLOCK)[:, :N]
    return codes.contiguous(), byte


def _as_values(codes, byte):
    return {"values": codes.view(torch.float8_e4m3fn), "scales": byte.view(torch.float8_e8m0fnu)}


def _plain_norm(s):
    case = s["case"]
    h = s["x"].float()
    out = {}
    if case["residual"]:
        h = h + s["residual"].float()
        out["sum"] = h.to(torch.bfloat16)
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
    out["y"] = y.to(torch.bfloat16) if case["out"] == "bf16" else _as_values(*_rows8(y))
    return out


def _plain_gemm8(s):
    case = s["case"]
    K, N = case["K"], case["N"]
    codes, byte = (s["x8"], s["x_scales"]) if case["x"] == "rows8" else _rows8(s["x"].float())
    x = codes.view(torch.float8_e4m3fn).float() * _pow2(byte).repeat_interleave(BLOCK, 1)[:, :K]
    w = s["w"].view(torch.float8_e4m3fn).float() * s["w_scales"].repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]
    return torch.matmul(x, w.t()).to(torch.bfloat16)


def _token_rows(s):
    """(sequence, position) of every new token."""
    b = s["batch"]
    offsets = b["offsets"].long()
    t = torch.arange(b["T"], device="cuda")
    seq = torch.searchsorted(offsets[1:], t, right=True)
    return seq, b["kv"].long()[seq] - offsets[seq + 1] + t


def _rotate(x, table, rot, pairs):
    """x fp32 [T][H][D] with the first `rot` dimensions rotated by table fp32 [T][rot]."""
    c, n = table[:, None, : rot // 2], table[:, None, rot // 2:]
    if pairs == "half":
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        r = torch.cat((a * c - b * n, b * c + a * n), -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack((a * c - b * n, b * c + a * n), -1).flatten(-2)
    return torch.cat((r, x[..., rot:]), -1)


def _plain_append(s):
    case, b, c = s["case"], s["batch"], s["cache"]
    P, pages, Hkv = case["P"], b["pages"], case["Hkv"]
    seq, pos = _token_rows(s)
    table = s["rope"][pos]
    q = _rotate(s["q"].float(), table, case["rot"], case["pairs"]).to(torch.bfloat16)
    page, slot = b["table"].long()[seq, pos // P], pos % P
    # the one page of each sequence that may hold older tokens
    old = b["kv"].long() - (b["offsets"][1:] - b["offsets"][:-1]).long()
    part = b["table"].long().gather(1, (old // P).clamp(max=b["table"].shape[1] - 1)[:, None])[:, 0]
    older = torch.arange(P, device="cuda") < (old % P)[:, None]
    for name, new, axis in (("k", _rotate(s["k"].float(), table, case["rot"], case["pairs"]), 2), ("v", s["v"].float(), 3)):
        codes, byte = c[name], c[name + "_scales"]
        amax = torch.zeros((pages, Hkv), device="cuda").index_reduce_(0, page, new.abs().amax(2), "amax")
        fresh = _exponent(amax, -CACHE_EXP, CACHE_EXP)
        touched = torch.zeros(pages, dtype=torch.bool, device="cuda").index_fill_(0, page, True)
        kept = torch.zeros(pages, dtype=torch.bool, device="cuda").index_put_((part,), (old % P > 0) & (old < b["kv"]))
        scale = torch.where(touched[:, None], torch.where(kept[:, None], torch.maximum(fresh, byte), fresh), byte)
        was = codes[part]
        moved = (was.view(torch.float8_e4m3fn).float() * torch.exp2(byte[part].float() - scale[part].float())[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        mine = older[:, None, :, None] if axis == 2 else older[:, None, None, :]
        codes[part] = torch.where(mine, moved, was)
        byte.copy_(scale)
        bytes_new = (new / _pow2(scale[page])[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        if axis == 2:
            codes[page, :, slot] = bytes_new
        else:
            codes[page, :, :, slot] = bytes_new
    return {"q": q, "k": _as_values(c["k"], c["k_scales"]), "v": _as_values(c["v"], c["v_scales"])}


def _plain_attention(s):
    case, b, c = s["case"], s["batch"], s["cache"]
    B, n, Hkv, D, P = case["B"], case["n"], case["Hkv"], case["D"], case["P"]
    G, L = case["Hq"] // case["Hkv"], b["table"].shape[1] * P
    at = b["table"].clamp(min=0).long()
    kv = b["kv"].long()
    there = torch.arange(L, device="cuda") < kv[:, None]
    k = c["k"][at].view(torch.float8_e4m3fn).float() * _pow2(c["k_scales"][at])[..., None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(B, Hkv, D, L)
    v = c["v"][at].view(torch.float8_e4m3fn).float() * _pow2(c["v_scales"][at])[..., None, None]
    v = torch.where(there[:, None, :, None], v.permute(0, 2, 1, 4, 3).reshape(B, Hkv, L, D), 0.0)
    seq, pos = _token_rows(s)
    row = torch.arange(b["T"], device="cuda") - b["offsets"].long()[seq]
    q = torch.zeros((B, n, Hkv, G, D), device="cuda")
    q[seq, row] = s["q"].float().view(-1, Hkv, G, D)
    scores = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D), k).view(B, Hkv, G, n, L) * (D ** -0.5)
    where = torch.full((B, n), -1, dtype=torch.int64, device="cuda")
    where[seq, row] = pos
    j = torch.arange(L, device="cuda")
    seen = (j <= where[..., None]) & there[:, None, :]
    if case["window"]:
        seen &= j > where[..., None] - case["window"]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, G * n, L), v).view(B, Hkv, G, n, D) / torch.where(total > 0, total, 1.0)
    return o.permute(0, 3, 1, 2, 4)[seq, row].reshape(-1, case["Hq"], D).to(torch.bfloat16)


# ---- the calls -----------------------------------------------------------------------------------------------------------

def _own(s):
    from paper_2507_07145_amd import layer
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        res = {"residual": s["residual"], "residual_out": s["sum"]} if case["residual"] else {}
        y = layer.rms_norm(s["x"], s["weight"], EPS, rows8=case["out"] == "rows8", **res)
        out = {"sum": s["sum"]} if case["residual"] else {}
        out["y"] = y if case["out"] == "bf16" else _as_values(y.codes, y.scales)
        return out
    if kind == "gemm8":
        return layer.gemm8(s["own_w"], s["own_x"] if case["x"] == "rows8" else s["x"])
    if kind == "append":
        c = s["cache"]
        q = layer.cache_append(s["own_cache"], s["own_batch"], s["k"], s["v"], q=s["q"], rope=s["own_rope"])
        return {"q": q, "k": _as_values(c["k"], c["k_scales"]), "v": _as_values(c["v"], c["v_scales"])}
    return layer.attention(s["own_cache"], s["own_batch"], s["q"], window=case["window"])


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "gemm8": _plain_gemm8, "append": _plain_append, "attention": _plain_attention}[state["case"]["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def _seen(p, length, window):
    """Cached tokens that position p of a sequence of `length` sees."""
    last = min(p, length - 1)
    first = max(0, p - window + 1) if window else 0
    return max(0, last - first + 1)


def work(case):
    kind = case["kind"]
    if kind == "norm":
        M, N = case["M"], case["N"]
        wide = 2 if case["out"] == "bf16" else 1 + 1 / BLOCK
        return {"bytes": int(M * N * (2 + (4 if case["residual"] else 0) + wide) + 2 * N), "flops": 5 * M * N}
    if kind == "gemm8":
        M, K, N = case["M"], case["K"], case["N"]
        x = M * K * (1 + 1 / BLOCK) if case["x"] == "rows8" else 2 * M * K
        return {"bytes": int(K * N + 4 * K * N / BLOCK ** 2 + x + 2 * M * N), "flops": 2 * M * K * N}
    new, lens = _lengths(case)
    T, row = sum(new), case["Hkv"] * case["D"]
    q = 2 * T * case["Hq"] * case["D"]
    if kind == "append":
        return {"bytes": int(2 * q + T * row * (4 + 2) + 4 * T * case["rot"]), "flops": 3 * T * case["rot"] * (case["Hq"] + case["Hkv"])}
    cached = pairs = 0
    for n, length in zip(new, lens):
        first = max(0, length - n - case["window"] + 1) if case["window"] else 0
        cached += length - first
        pairs += sum(_seen(p, length, case["window"]) for p in range(length - n, length))
    return {"bytes": int(2 * q + cached * row * 2 + 2 * cached // case["P"] * case["Hkv"]), "flops": 4 * pairs * case["Hq"] * case["D"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _value(codes):
    return codes.view(torch.float8_e4m3fn).double()


def _step(amax, lo):
    """The power of two that a block whose largest magnitude is amax (64 bits) is held in units of."""
    e = torch.ceil(torch.log2(torch.clamp(amax, min=1e-300) / E4M3_MAX))
    e = torch.where(amax > E4M3_MAX * torch.exp2(e), e + 1, torch.where(amax <= E4M3_MAX * torch.exp2(e - 1), e - 1, e))
    return torch.exp2(e.clamp(min=lo))


def _exact_norm(case, s):
    h = s["x"].double() + (s["residual"].double() if case["residual"] else 0.0)
    y = s["weight"].double() * h / (h.square().sum(1, keepdim=True) / case["N"] + EPS).sqrt()
    out = {"sum": h} if case["residual"] else {}
    if case["out"] == "bf16":
        out["y"] = y
    else:   # the numbers that the 8 bits are nearest to
        pieces = torch.split(y, BLOCK, 1)
        steps = [_step(p.abs().amax(1, keepdim=True), -126) for p in pieces]
        out["y"] = {"values": torch.cat([p / t for p, t in zip(pieces, steps)], 1), "scales": torch.cat(steps, 1)}
    return out


def _exact_gemm8(case, s):
    M, K, N = case["M"], case["K"], case["N"]
    y = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    for i, k in enumerate(range(0, K, BLOCK)):
        if case["x"] == "rows8":
            x = _value(s["x8"][:, k:k + BLOCK].contiguous()) * torch.exp2(s["x_scales"][:, i:i + 1].double() - 127)
        else:
            x = s["x"][:, k:k + BLOCK].double()
            t = _step(x.abs().amax(1, keepdim=True), -126)
            x = (x / t).float().to(torch.float8_e4m3fn).double() * t
        w = _value(s["w"][:, k:k + BLOCK].contiguous())
        by_row = s["w_scales"][torch.arange(N, device="cuda") // BLOCK, i].double()
        y += (x @ w.t().contiguous()) * by_row
    return y


def _exact_append(case, s):
    b, c, P, rot = s["batch"], s["cache"], case["P"], case["rot"]
    half = rot // 2
    i = torch.arange(half, device="cuda")
    first, second = (i, i + half) if case["pairs"] == "half" else (2 * i, 2 * i + 1)
    values = {"k": _value(c["k"]), "v": _value(c["v"]).transpose(2, 3)}
    scales = {m: torch.exp2(c[m + "_scales"].double() - 127) for m in ("k", "v")}
    q_out, at = torch.empty_like(s["q"], dtype=torch.float64), 0
    for seq, (n, length) in enumerate(zip(b["n"], b["lens"])):
        rows = slice(at, at + n)
        at += n
        table = s["rope"][length - n:length].double()[:, None]
        turned = []
        for x in (s["q"][rows].double(), s["k"][rows].double()):
            z = x.clone()
            z[..., first] = x[..., first] * table[..., :half] - x[..., second] * table[..., half:]
            z[..., second] = x[..., second] * table[..., :half] + x[..., first] * table[..., half:]
            turned.append(z)
        q_out[rows] = turned[0]
        for m, new in (("k", turned[1]), ("v", s["v"][rows].double())):
            for w in range((length - n) // P, (length - 1) // P + 1):
                page = int(b["table"][seq, w])
                lo, hi = max(length - n, w * P), min(length, (w + 1) * P)
                tokens = new[lo - (length - n):hi - (length - n)]
                step = _step(tokens.abs().amax((0, 2)), -CACHE_EXP)
                if lo > w * P:
                    grown = torch.maximum(step, scales[m][page])
                    values[m][page][:, :lo - w * P] *= (scales[m][page] / grown)[:, None, None]
                    step = grown
                scales[m][page] = step
                values[m][page][:, lo - w * P:hi - w * P] = tokens.transpose(0, 1) / step[:, None, None]
    return {"q": q_out, "k": {"values": values["k"], "scales": scales["k"]}, "v": {"values": values["v"].transpose(2, 3), "scales": scales["v"]}}


def _exact_attention(case, s):
    b, c, D, G = s["batch"], s["cache"], case["D"], case["Hq"] // case["Hkv"]
    out, at = torch.zeros_like(s["q"], dtype=torch.float64), 0
    for seq, (n, length) in enumerate(zip(b["n"], b["lens"])):
        pages = b["table"][seq, :-(-length // case["P"])].long()
        k = (_value(c["k"][pages]) * torch.exp2(c["k_scales"][pages].double() - 127)[..., None, None]).transpose(0, 1).flatten(1, 2)[:, :length]
        v = (_value(c["v"][pages]) * torch.exp2(c["v_scales"][pages].double() - 127)[..., None, None]).permute(1, 0, 3, 2).flatten(1, 2)[:, :length]
        age = torch.arange(length - n, length, device="cuda")[:, None] - torch.arange(length, device="cuda")
        hidden = (age < 0) | (age >= case["window"] if case["window"] else age < 0)
        for h in range(case["Hq"]):
            x = (s["q"][at:at + n, h].double() @ k[h // G].t().contiguous()) / math.sqrt(D)
            out[at:at + n, h] = torch.softmax(x.masked_fill_(hidden, -math.inf), 1) @ v[h // G].contiguous()
        at += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "gemm8": _exact_gemm8, "append": _exact_append, "attention": _exact_attention}[case["kind"]](case, s)
