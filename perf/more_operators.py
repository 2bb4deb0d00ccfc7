"""Rows that choose their weights, as a serving program calls the operators around the 2-bit grouped products and beside the shared ones.

Four kinds of case, through the public functions of `paper_2507_07145_amd.routing`:

  route      logits of a router to experts and weights (softmax or sigmoid scores, a bias that takes part in the choice alone, groups of experts of
             which the best are kept, top k, renormalised weights), with the order of rows that `binding.grouped_gemm` reads.
  sort       that order for ids that are there already: the experts of one GPU's share, the adapters of a batch's requests.
  combine    y[t] = base[t] + sum over j of weights[t][j] rows[places[t][j]]: the end of a layer of experts.
  adapters   out[t] = y[t] + scales[a] (x[t] A[a]^T) B[a]^T, a the adapter of row t's request, beside a projection that all requests share.

An order: the entries (t, j) sorted by id, then t, then j, those whose id is none of `experts` experts from `first` on after all others: `rows` their t, `experts`
their id - first (-1: none); `offsets` where each expert's begin and the last one's end; `places` [T][k] where each entry went (-1: none).
"""
import math
import random

import torch

own = False

# the largest of each kind: what draw() stays below
MAX_LOGITS = 16384 * 256
MAX_ENTRIES = 16384 * 8
MAX_COMBINE = 2048 * 8 * 7168
MAX_ADAPTER_ROWS = 2048 * (7168 + 18432)
MAX_ADAPTER_WEIGHTS = 96 * 32 * (4096 + 11008)
MAX_ADAPTER_PRODUCTS = 2048 * 64 * (7168 + 18432)


def listed():
    return [
        # one token, a router's plain softmax: launch and call overhead
        {"name": "route-1x64", "kind": "route", "T": 1, "E": 64, "k": 8, "scoring": "softmax", "bias": False, "G": 1, "g": 1, "best": 1, "renorm": True, "scale": 1.0, "type": "bf16", "pad": 0},
        # a decode batch padded for a captured graph: sigmoid scores, balance bias, groups
        {"name": "route-64x256", "kind": "route", "T": 64, "E": 256, "k": 8, "scoring": "sigmoid", "bias": True, "G": 8, "g": 4, "best": 2, "renorm": True, "scale": 2.5, "type": "fp32", "pad": 5},
        # a short prompt, numbers that are no powers of two, groups by their best expert
        {"name": "route-511x160", "kind": "route", "T": 511, "E": 160, "k": 6, "scoring": "softmax", "bias": False, "G": 8, "g": 3, "best": 1, "renorm": False, "scale": 16.0, "type": "bf16", "pad": 0},
        # prompts of a full step
        {"name": "route-16384x256", "kind": "route", "T": 16384, "E": 256, "k": 8, "scoring": "sigmoid", "bias": True, "G": 8, "g": 4, "best": 2, "renorm": True, "scale": 2.5, "type": "fp32", "pad": 0},
        # the adapters of a decode batch's requests, some without one
        {"name": "sort-200of128", "kind": "sort", "T": 200, "k": 1, "experts": 128, "E": 128, "first": 0, "none": 0.2},
        # one GPU's quarter of the experts, prompts of a full step
        {"name": "sort-16384x8", "kind": "sort", "T": 16384, "k": 8, "experts": 256, "E": 64, "first": 64, "none": 0.0},
        # one token's eight experts
        {"name": "combine-1x7168", "kind": "combine", "T": 1, "k": 8, "N": 7168, "E": 64, "base": True, "none": 0.0},
        # a prompt, added to what the shared expert gave
        {"name": "combine-2048x7168", "kind": "combine", "T": 2048, "k": 8, "N": 7168, "E": 64, "base": True, "none": 0.0},
        # one token of one request through a square projection
        {"name": "adapters-1x8192", "kind": "adapters", "T": 1, "K": 8192, "N": 8192, "R": 16, "n": 8, "none": 0.0, "ranks": False, "chunks": False},
        # a decode batch, ragged in every dimension, several ranks, some requests without an adapter
        {"name": "adapters-37x7184", "kind": "adapters", "T": 37, "K": 7184, "N": 5001, "R": 24, "n": 12, "none": 0.2, "ranks": True, "chunks": False},
        # a large decode batch of nearly as many requests' adapters
        {"name": "adapters-128x4096", "kind": "adapters", "T": 128, "K": 4096, "N": 11008, "R": 32, "n": 96, "none": 0.0, "ranks": True, "chunks": False},
        # prompts of four requests, up projection
        {"name": "adapters-2048x7168", "kind": "adapters", "T": 2048, "K": 7168, "N": 18432, "R": 64, "n": 4, "none": 0.0, "ranks": False, "chunks": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "route", "sort", "combine", "adapters", "adapters"])
    while True:
        if kind == "route":
            G = rng.choice((1, 1, 2, 4, 8))
            E = G * _log(rng, 8, 512 // G)
            g = rng.randint(max(1, G // 3), G)
            case = {"T": _log(rng, 1, 32768), "E": E, "k": rng.choice((1, 2, 4, 6, 8, 8)), "scoring": rng.choice(("softmax", "sigmoid")), "bias": rng.random() < 0.5, "G": G, "g": g,
                    "best": rng.choice((1, 2)), "renorm": rng.random() < 0.6, "scale": rng.choice((1.0, 2.5)), "type": rng.choice(("bf16", "fp32"))}
            case["pad"] = rng.choice((0, 0, case["T"] // 8))
            fits = case["T"] * E <= MAX_LOGITS and case["T"] * case["k"] <= MAX_ENTRIES
        elif kind == "sort":
            experts = _log(rng, 4, 1024)
            E = rng.choice((experts, max(1, experts // 4)))
            case = {"T": _log(rng, 1, 65536), "k": rng.choice((1, 1, 2, 6, 8)), "experts": experts, "E": E, "first": rng.choice((0, experts - E)), "none": rng.choice((0.0, 0.3))}
            case["k"] = min(case["k"], experts)
            fits = case["T"] * case["k"] <= MAX_ENTRIES and case["T"] * experts <= MAX_LOGITS * 4
        elif kind == "combine":
            case = {"T": _log(rng, 1, 8192), "k": rng.choice((1, 2, 6, 8)), "N": _log(rng, 500, 8192), "E": _log(rng, 8, 256), "base": rng.random() < 0.6, "none": rng.choice((0.0, 0.25))}
            if rng.random() < 0.6:
                case["N"] = case["N"] // 64 * 64 + 64
            fits = case["T"] * case["k"] * case["N"] <= MAX_COMBINE
        else:
            case = {"T": _log(rng, 1, 4096), "K": 8 * _log(rng, 64, 2304), "N": _log(rng, 500, 18432), "R": rng.choice((8, 16, 16, 32, 64, 128)), "n": _log(rng, 1, 128),
                    "none": rng.choice((0.0, 0.25)), "ranks": rng.random() < 0.5, "chunks": rng.random() < 0.5}
            if rng.random() < 0.5:
                case["K"], case["N"] = (case["K"] + 63) // 64 * 64, (case["N"] + 63) // 64 * 64
            fits = case["T"] * (case["K"] + case["N"]) <= MAX_ADAPTER_ROWS and case["n"] * case["R"] * (case["K"] + case["N"]) <= MAX_ADAPTER_WEIGHTS \
                and case["T"] * case["R"] * (case["K"] + case["N"]) <= MAX_ADAPTER_PRODUCTS
        if fits:
            return {"kind": kind, **case}


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 16 + stream) & (2 ** 62 - 1))


def _normal(shape, seed, stream, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=_gen(seed, stream))


def _uniform(shape, seed, stream):
    return torch.rand(shape, device="cuda", generator=_gen(seed, stream))


def _distinct(T, experts, k, seed, stream):
    """k different experts of each row, popular ones more often."""
    liking = _normal((T, experts), seed, stream) + _normal((1, experts), seed, stream + 1, 0.5)
    return liking.topk(k, 1).indices.to(torch.int32)


def _adapter_ids(case):
    """The adapter of each row (-1: none): one to a chunk of rows, as prompts of several requests have it, or at random.  Sizes and adapters in use go by the
    case alone, so that its work is the same for every seed."""
    r = random.Random(case["T"] * 1000003 + case["K"] * 101 + case["n"])
    T, n = case["T"], case["n"]
    pick = lambda: -1 if r.random() < case["none"] else r.randrange(n)  # noqa: E731
    if not case["chunks"]:
        return [pick() for _ in range(T)]
    cuts = sorted(r.randrange(T + 1) for _ in range(min(n, 8) - 1))
    ids, order = [], list(range(n))
    r.shuffle(order)
    for i, (a, b) in enumerate(zip([0] + cuts, cuts + [T])):
        ids += [-1 if r.random() < case["none"] else order[i]] * (b - a)
    return ids


def _ranks(case):
    r = random.Random(case["K"] * 31 + case["N"])
    return [case["R"]] + [r.choice((case["R"], case["R"], max(4, case["R"] // 2), r.randint(1, case["R"]))) for _ in range(case["n"] - 1)]


def prepare(case, seed):
    s = {"case": case}
    kind = case["kind"]
    if kind == "route":
        logits = _normal((case["T"], case["E"]), seed, 0, 1.5) + _normal((1, case["E"]), seed, 1, 0.5)
        if case["pad"]:
            logits[case["T"] - case["pad"]:] = -math.inf
        s["logits"] = logits.to(torch.bfloat16) if case["type"] == "bf16" else logits
        s["bias"] = _normal((case["E"],), seed, 2, 0.1) if case["bias"] else None
    elif kind == "sort":
        s["ids"] = _distinct(case["T"], case["experts"], case["k"], seed, 0)
        if case["none"]:
            s["ids"][_uniform(s["ids"].shape, seed, 2) < case["none"]] = -1
    elif kind == "combine":
        T, k = case["T"], case["k"]
        ids = _distinct(T, max(case["E"], k), k, seed, 0)
        if case["none"]:
            ids[_uniform((T, k), seed, 2) < case["none"]] = -1
        s["places"] = _plain_order(ids, 0, max(case["E"], k))["places"]
        s["weights"] = torch.softmax(_normal((T, k), seed, 3), 1)
        s["rows"] = _normal((T * k, case["N"]), seed, 4).to(torch.bfloat16)
        s["base"] = _normal((T, case["N"]), seed, 5).to(torch.bfloat16) if case["base"] else None
    else:
        T, K, N, R, n = (case[m] for m in ("T", "K", "N", "R", "n"))
        s["x"] = _normal((T, K), seed, 0).to(torch.bfloat16)
        s["y"] = _normal((T, N), seed, 1).to(torch.bfloat16)
        s["A"] = _normal((n, R, K), seed, 2, K ** -0.5).to(torch.bfloat16)
        s["B"] = _normal((n, N, R), seed, 3, 0.3 * R ** -0.5).to(torch.bfloat16)
        s["scales"] = 0.5 + _uniform((n,), seed, 4)
        s["ranks"] = torch.tensor(_ranks(case), dtype=torch.int32, device="cuda") if case["ranks"] else None
        ids = torch.tensor(_adapter_ids(case), dtype=torch.int32, device="cuda")[:, None]
        s["order"] = _plain_order(ids, 0, n)   # one a step, for all projections of all layers
        if own:   # the handles that a program makes once and keeps
            from paper_2507_07145_amd import routing
            s["own_adapters"] = routing.Adapters(s["A"], s["B"], scales=s["scales"], ranks=s["ranks"])
            s["own_order"] = routing.Order(**s["order"])
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------

def _plain_order(ids, first, E):
    T, k = ids.shape
    flat = ids.reshape(-1).long() - first
    flat = torch.where((flat >= 0) & (flat < E), flat, E)
    key, entry = torch.sort(flat, stable=True)
    here = key < E
    places = torch.empty_like(flat)
    places[entry] = torch.where(here, torch.arange(T * k, device=ids.device), -1)
    offsets = torch.searchsorted(key, torch.arange(E + 1, device=ids.device))
    whole = lambda v: v.to(torch.int32)  # noqa: E731
    return {"rows": whole(entry // k), "experts": whole(torch.where(here, key, -1)), "offsets": whole(offsets), "places": whole(places.view(T, k))}


def _plain_route(s):
    """Scores in 64 bits: experts next to a border change places with the last bits."""
    case, bias = s["case"], s["bias"]
    T, E, k, G = case["T"], case["E"], case["k"], case["G"]
    l = s["logits"].double()
    open_ = l > -math.inf
    if case["scoring"] == "softmax":
        top = l.amax(1, keepdim=True).clamp(min=-1e300)
        e = torch.exp(l - top)
        score = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        score = 1.0 / (1.0 + torch.exp(-l))
    by = score + bias.double() if bias is not None else score
    by = torch.where(open_, by, -math.inf)
    one = by if bias is not None else l           # (without a bias the logits have the scores' order)
    if G > 1:
        best = by.view(T, G, E // G).topk(min(case["best"], E // G), 2).values
        value = torch.where(best[..., 0] > -math.inf, torch.where(best > -math.inf, best, 0.0).sum(2), -math.inf)
        kept = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :case["g"]]
        in_group = torch.zeros((T, G), dtype=torch.bool, device=l.device).scatter_(1, kept, True)
        one = torch.where(in_group.repeat_interleave(E // G, 1), one, -math.inf)
    one, ids = torch.sort(one, dim=1, descending=True, stable=True)
    one, ids = one[:, :k], ids[:, :k]
    w = torch.where(one > -math.inf, score.gather(1, ids), 0.0)
    ids = torch.where(one > -math.inf, ids, -1).to(torch.int32)
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return {"ids": ids, "weights": (w * case["scale"]).float(), **_plain_order(ids, 0, E)}


def _plain_combine(s):
    places = s["places"].long()
    w = torch.where(places >= 0, s["weights"], 0.0)
    rows = s["rows"][places.clamp(min=0)].float()
    y = (rows * w[..., None]).sum(1)
    if s["base"] is not None:
        y = y + s["base"].float()
    return y.to(torch.bfloat16)


def _plain_adapters(s):
    """Few rows: each with its adapter's matrices.  Many: products with all adapters at once, of which each row keeps its own."""
    case, order = s["case"], s["order"]
    T, K, N, R, n = (case[m] for m in ("T", "K", "N", "R", "n"))
    places = order["places"][:, 0].long()
    a = torch.where(places >= 0, order["experts"][places.clamp(min=0)].long(), -1)
    has = torch.arange(R, device="cuda") < (s["ranks"][:, None] if s["ranks"] is not None else R)      # [n or 1][R]
    factor = s["scales"][:, None] * has
    x = s["x"].float()
    if T < n:
        at = a.clamp(min=0)
        v = torch.matmul(s["A"][at].float(), x[:, :, None])[:, :, 0] * factor[at] * (a >= 0)[:, None]
        d = torch.matmul(s["B"][at].float(), v[:, :, None])[:, :, 0]
    else:
        v = torch.matmul(x, s["A"].float().view(n * R, K).t()).view(T, n, R) * factor
        v = v * (a[:, None] == torch.arange(n, device="cuda"))[:, :, None]
        d = torch.matmul(v.view(T, n * R), s["B"].float().transpose(1, 2).reshape(n * R, N))
    return (s["y"].float() + d).to(torch.bfloat16)


# ---- the calls -----------------------------------------------------------------------------------------------------------

def _own(s):
    from paper_2507_07145_amd import routing
    case, kind = s["case"], s["case"]["kind"]
    parts = lambda o: {"rows": o.rows, "experts": o.experts, "offsets": o.offsets, "places": o.places}  # noqa: E731
    if kind == "route":
        r = routing.route(s["logits"], case["k"], scoring=case["scoring"], bias=s["bias"], groups=case["G"], top_groups=case["g"], group_best=case["best"],
                          renormalize=case["renorm"], scale=case["scale"])
        return {"ids": r.ids, "weights": r.weights, **parts(r.order)}
    if kind == "sort":
        return parts(routing.sort_rows(s["ids"], case["E"], first=case["first"]))
    if kind == "combine":
        return routing.combine(s["rows"], s["places"], s["weights"], base=s["base"])
    return routing.adapters(s["y"], s["x"], s["own_adapters"], s["own_order"])


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["kind"] == "sort":
        return _plain_order(state["ids"], case["first"], case["E"])
    return {"route": _plain_route, "combine": _plain_combine, "adapters": _plain_adapters}[case["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    kind, T = case["kind"], case["T"]
    if kind == "route":
        entries = T * case["k"]
        return {"bytes": T * case["E"] * (2 if case["type"] == "bf16" else 4) + entries * 20 + 4 * case["E"], "flops": 8 * T * case["E"]}
    if kind == "sort":
        entries = T * case["k"]
        return {"bytes": entries * 16 + 4 * case["E"], "flops": entries}
    if kind == "combine":
        have = T * case["k"] * (1.0 - case["none"])
        return {"bytes": int(2 * case["N"] * (have + T * (2 if case["base"] else 1)) + 8 * T * case["k"]), "flops": int(2 * have * case["N"])}
    K, N = case["K"], case["N"]
    ids = _adapter_ids(case)
    rank = _ranks(case) if case["ranks"] else [case["R"]] * case["n"]
    rows = [a for a in ids if a >= 0]
    weights = sum(rank[a] for a in set(rows)) * (K + N)
    return {"bytes": 2 * (len(rows) * K + 2 * T * N + weights), "flops": sum(2 * rank[a] * (K + N) for a in rows)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _exact_order(ids, first, E):
    """A list of entries for each expert, and one for those of none, one after the other."""
    T, k = ids.shape
    local = ids.cpu().reshape(-1).to(torch.int64) - first
    lists = [[] for _ in range(E + 1)]
    for i, e in enumerate(local.tolist()):
        lists[e if 0 <= e < E else E].append(i)
    rows, experts, places, offsets = [], [], [-1] * (T * k), [0]
    for e, one in enumerate(lists):
        for i in one:
            if e < E:
                places[i] = len(rows)
            rows.append(i // k)
            experts.append(e if e < E else -1)
        if e < E:
            offsets.append(len(rows))
    whole = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return {"rows": whole(rows), "experts": whole(experts), "offsets": whole(offsets), "places": whole(places).view(T, k)}


def _exact_route(case, s):
    l = s["logits"].double().cpu()
    T, E, k, G = case["T"], case["E"], case["k"], case["G"]
    closed = torch.isneginf(l)
    if case["scoring"] == "softmax":
        score = torch.exp(l - torch.logsumexp(l, 1, keepdim=True)).nan_to_num(nan=0.0)
    else:
        score = torch.sigmoid(l)
    by = (score + (s["bias"].double().cpu() if case["bias"] else 0.0)).masked_fill(closed, -math.inf)
    left = (by if case["bias"] else l).clone()
    row = torch.arange(T)
    if G > 1:
        groups = by.view(T, G, E // G)
        first = groups.amax(2)
        value = first.clone()
        if case["best"] == 2 and E // G > 1:
            rest = groups.clone().scatter_(2, groups.argmax(2, keepdim=True), -math.inf).amax(2)
            value = value + torch.where(torch.isneginf(rest), 0.0, rest)
        taken = torch.zeros((T, G), dtype=torch.bool)
        for _ in range(case["g"]):
            at = _first_largest(value.masked_fill(taken, -math.inf), taken)
            taken[row, at] = True
        left.view(T, G, E // G).masked_fill_(~taken[..., None], -math.inf)
    ids, w = torch.full((T, k), -1), torch.zeros((T, k), dtype=torch.float64)
    for j in range(k):
        at = _first_largest(left, None)
        there = ~torch.isneginf(left[row, at])
        ids[:, j] = torch.where(there, at, -1)
        w[:, j] = torch.where(there, score[row, at], 0.0)
        left[row, at] = -math.inf
    if case["renorm"]:
        w /= w.sum(1, keepdim=True).clamp(min=1e-300)
    ids = ids.to(torch.int32)
    return {"ids": ids, "weights": w * case["scale"], **_exact_order(ids, 0, E)}


def _first_largest(v, closed):
    """Index of the first of each row's largest values (of those that are not closed)."""
    is_top = v == v.amax(1, keepdim=True)
    if closed is not None:
        is_top &= ~closed
    return (is_top.cumsum(1) == 0).sum(1).clamp(max=v.shape[1] - 1)


def _exact_combine(case, s):
    y = s["base"].double() if case["base"] else torch.zeros((case["T"], case["N"]), dtype=torch.float64, device="cuda")
    for j in range(case["k"]):
        at = s["places"][:, j].long()
        some = (at >= 0).nonzero()[:, 0]
        y[some] += s["weights"][some, j, None].double() * s["rows"][at[some]].double()
    return y


def _exact_adapters(case, s):
    y = s["y"].double()
    rank = _ranks(case) if case["ranks"] else [case["R"]] * case["n"]
    ids = torch.tensor(_adapter_ids(case), device="cuda")
    for a in sorted(set(ids.tolist()) - {-1}):
        t = (ids == a).nonzero()[:, 0]
        v = s["x"][t].double() @ s["A"][a, :rank[a]].double().t().contiguous()
        y[t] += float(s["scales"][a]) * (v @ s["B"][a, :, :rank[a]].double().t().contiguous())
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sort":
        return _exact_order(s["ids"], case["first"], case["E"])
    return {"route": _exact_route, "combine": _exact_combine, "adapters": _exact_adapters}[case["kind"]](case, s)
