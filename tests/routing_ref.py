"""The operators of routing.py in 64 bits on the CPU, one row after the other, written from their definitions."""
import math

import numpy as np

U24 = 2.0 ** -24     # half a step of fp32, relative
U8 = 2.0 ** -8       # of bf16


def scores(l, scoring):
    """fp64 scores of one row of logits (fp64; NaN counts as -infinity)."""
    l = np.where(np.isnan(l), -np.inf, l)
    if scoring == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-l))
    top = l.max()
    if top == -np.inf:
        return np.zeros_like(l)
    with np.errstate(invalid="ignore"):
        e = np.where(l == top, 1.0, np.where(l == -np.inf, 0.0, np.exp(l - top)))
    return e / e.sum()


def best_first(values, n):
    """Indices of the n largest, the largest first, equal ones by the lower index."""
    return sorted(range(len(values)), key=lambda i: (-values[i], i))[:n]


def route(logits, k, scoring="softmax", bias=None, groups=1, top_groups=None, group_best=2, renormalize=False, scale=1.0):
    """ids [T][k], weights fp64 [T][k] of fp64 logits [T][E]."""
    T, E = logits.shape
    top_groups = groups if top_groups is None else top_groups
    ids, weights = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    size = E // groups
    for t in range(T):
        l, s = logits[t], scores(logits[t], scoring)
        is_open = ~(np.isnan(l) | (l == -np.inf))
        by = s.copy()
        if bias is not None:
            is_open &= ~(np.isnan(bias) | (bias == -np.inf))
            by = s + np.where(np.isnan(bias), 0.0, bias)
        kept = range(groups)
        if top_groups < groups:
            value = []
            for g in range(groups):
                have = sorted((by[e] for e in range(g * size, (g + 1) * size) if is_open[e]), reverse=True)[:group_best]
                value.append(sum(have) if have else -math.inf)
            kept = best_first(value, top_groups)
        left = [e for g in kept for e in range(g * size, (g + 1) * size) if is_open[e]]
        key = by if bias is not None else l
        chosen = sorted(left, key=lambda e: (-key[e], e))[:k]
        w = s[chosen]
        if renormalize:
            w = w / w.sum() if w.sum() > 0 else np.zeros_like(w)
        ids[t, :len(chosen)] = chosen
        weights[t, :len(chosen)] = w * scale
    return ids, weights


def order(ids, experts, first=0):
    """rows, experts, offsets, places of ids [T][k]."""
    T, k = ids.shape
    local = [int(i) - first for i in ids.reshape(-1)]
    local = [e if 0 <= e < experts else experts for e in local]
    at = sorted(range(T * k), key=lambda i: (local[i], i))
    places = [-1] * (T * k)
    for p, i in enumerate(at):
        if local[i] < experts:
            places[i] = p
    offsets = [sum(1 for e in local if e < x) for x in range(experts + 1)] if experts <= 64 else np.concatenate([[0], np.bincount(local, minlength=experts + 1)[:experts].cumsum()]).tolist()
    return (np.array([i // k for i in at], dtype=np.int64), np.array([local[i] if local[i] < experts else -1 for i in at], dtype=np.int64), np.array(offsets, dtype=np.int64),
            np.array(places, dtype=np.int64).reshape(T, k))


def combine(rows, places, weights, base=None):
    """(sums, how far fp32 sums may be off them) in fp64."""
    T, k = places.shape
    y = np.zeros((T, rows.shape[1])) if base is None else base.astype(np.float64).copy()
    size = np.abs(y)
    for t in range(T):
        for j in range(k):
            p = places[t, j]
            if 0 <= p < rows.shape[0]:
                y[t] += weights[t, j] * rows[p]
                size[t] += np.abs(weights[t, j] * rows[p])
    return y, (k + 1) * U24 * size


def adapters(y, x, a, b, ids, scales=None, ranks=None):
    """(results, how far fp32 sums and the second product's operand may be off) in fp64.  A sum of n terms in fp32 is off by at most n steps of 2^-23 of
    the terms' magnitudes, whatever its order and whether its additions round or cut off; x a^T enters the second product within 2^-15."""
    out, off = y.copy(), np.zeros_like(y)
    K = x.shape[1]
    for t, i in enumerate(ids):
        if not 0 <= i < a.shape[0]:
            continue
        r = a.shape[1] if ranks is None else min(max(int(ranks[i]), 0), a.shape[1])
        s = 1.0 if scales is None else float(scales[i])
        A, B = a[i, :r], b[i, :, :r]
        v = A @ x[t]
        dv = (K + 34) * 2 * U24 * (np.abs(A) @ np.abs(x[t])) + 2.0 ** -15 * np.abs(v) * 1.01      # 32 partial sums and the scale's product on top
        out[t] += s * (B @ v)
        off[t] = abs(s) * (np.abs(B) @ (dv + (2 * r + 2) * 2 * U24 * np.abs(v))) + 2 * U24 * np.abs(y[t])
    return out, off


def near(got, want, off, what, half_step=U8):
    """got within `off` and the result's own rounding of want; NaN and infinities where want has them."""
    got = np.asarray(got, dtype=np.float64)
    plain = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN elsewhere"
    assert np.array_equal(got[~plain & ~np.isnan(want)], want[~plain & ~np.isnan(want)]), f"{what}: infinities elsewhere"
    got, want, off = (np.broadcast_to(v, plain.shape)[plain] for v in (got, want, off))
    far = np.abs(got - want) - (off + half_step * (np.abs(want) + off) + 2.0 ** -134)
    assert far.size == 0 or far.max() <= 0, f"{what}: {far.max()} too far"
