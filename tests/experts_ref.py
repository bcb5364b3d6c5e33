"""The expert operators in 64 bits on the CPU, row by row from their formulas: the references of the tests."""
import math

import numpy as np
import torch

INF = float("inf")


def scores(x, kind):
    """Scores of one row of logits (float64 numpy) and which experts are free."""
    free = x > -INF                       # a NaN is not
    s = np.zeros_like(x)
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            s[free] = 1.0 / (1.0 + np.exp(-x[free]))
    elif free.any():
        top = x[free].max()
        e = (x[free] == INF).astype(float) if top == INF else np.exp(x[free] - top)
        s[free] = e / e.sum()
    return s, free


def choose(x, kind, K, bias=None, groups=1, top_groups=1, group_best=1, renorm=False, scale=1.0):
    """ids and weights of one row."""
    x = np.asarray(x, np.float64)
    E = x.size
    s, free = scores(x, kind)
    c = s if bias is None else s + np.asarray(bias, np.float64)
    able = free & (c > -INF)
    size = E // groups
    value = []
    for g in range(groups):
        best = sorted((c[e] for e in range(g * size, (g + 1) * size) if able[e]), reverse=True)[:group_best]
        value.append(sum(best) if best else -INF)
    taken = sorted((g for g in range(groups) if value[g] > -INF), key=lambda g: (-value[g], g))[:top_groups]
    # without a bias and groups the order is that of the logits, of which the scores are a rising function
    key = x if bias is None and groups == 1 else c
    ids = sorted((e for e in range(E) if able[e] and e // size in taken), key=lambda e: (-key[e], e))[:K]
    w = [s[e] for e in ids]
    if renorm:
        total = math.fsum(w)
        w = [v / total if total > 0 else 0.0 for v in w]
    return ids + [-1] * (K - len(ids)), [v * scale for v in w] + [0.0] * (K - len(ids))


def weights_of(x, ids, kind, renorm, scale):
    """The weights of given choices as a differentiable function of a row of logits (torch float64)."""
    there = [e for e in ids if e >= 0]
    w = torch.zeros(len(ids), dtype=torch.float64)
    if not there:
        return w
    free = torch.isfinite(x)
    s = torch.sigmoid(x) if kind == "sigmoid" else torch.softmax(torch.where(free, x, torch.tensor(-INF).double()), 0)
    v = s[there]
    if renorm:
        v = v / v.sum()
    return torch.cat([v * scale, torch.zeros(len(ids) - len(there), dtype=torch.float64)])


def plan(ids, E):
    """offsets, order, slot of ids[n][K]."""
    flat = np.asarray(ids).reshape(-1)
    order = [p for e in range(E) for p in np.flatnonzero(flat == e)]
    offsets = np.concatenate([[0], np.cumsum([(flat == e).sum() for e in range(E)])]).astype(np.int32)
    slot = np.full(flat.size, -1, np.int32)
    slot[order] = np.arange(len(order))
    return offsets, np.asarray(order, np.int32), slot.reshape(np.asarray(ids).shape)


def philox4x32(counter, key):
    """Philox4x32-10 on python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def drop_limit(p):
    return round(65536.0 * (1.0 - float(np.float32(p))))


def drop_factor(rows, d, p, seed, step):
    """Factor of every element: 0 or the scale."""
    limit = drop_limit(p)
    key = (seed & 0xFFFFFFFF, seed >> 32)
    draws = np.zeros((rows, (d + 7) // 8 * 8), np.int64)
    for r in range(rows):
        for g in range((d + 7) // 8):
            words = philox4x32((g, r + 1, step & 0xFFFFFFFF, step >> 32), key)
            for i, w in enumerate(words):
                draws[r, 8 * g + 2 * i], draws[r, 8 * g + 2 * i + 1] = w & 0xFFFF, w >> 16
    kept = draws[:, :d] < limit
    return kept * (65536.0 / limit if limit else 0.0)


def silu(g):
    return g / (1.0 + np.exp(-g))


def silu_slope(g):
    z = 1.0 / (1.0 + np.exp(-g))
    return z + g * z * (1.0 - z)
