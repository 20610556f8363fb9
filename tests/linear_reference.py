"""Matrices in 4 bits, routing and turned rows from their definitions, in numpy and 64 bits (not collected by pytest)."""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ matrices in 4 bits

def brain_below(x):
    """float32 rounded down to bfloat16's values."""
    x = np.asarray(x, np.float32)
    cut = x.view(np.uint32) & np.uint32(0xffff0000)
    down = np.where((cut != x.view(np.uint32)) & (x < 0), cut + np.uint32(0x10000), cut).astype(np.uint32)
    return down.view(np.float32)


def quantise(weight, group):
    """Codes [N, K], scale and minimum [N, groups] of a matrix; steps in fp32."""
    w = np.asarray(weight, np.float32)
    N, K = w.shape
    groups = -(-K // group)
    codes = np.zeros((N, K), np.uint8)
    scale, low = np.zeros((N, groups), np.float32), np.zeros((N, groups), np.float32)
    with np.errstate(all="ignore"):
        for g in range(groups):
            part = w[:, g * group:(g + 1) * group]
            mn = brain_below(part.min(1))
            s = -brain_below(-((part.max(1) - mn).astype(np.float32) / np.float32(15)).astype(np.float32))
            bad = ~np.isfinite(part).all(1) | ~np.isfinite(mn) | ~np.isfinite(s)
            q = np.rint(((part - mn[:, None]).astype(np.float32) / s[:, None]).astype(np.float32))
            q = np.where((s > 0)[:, None] & ~bad[:, None], np.clip(np.nan_to_num(q), 0, 15), 0)
            codes[:, g * group:(g + 1) * group] = q
            scale[:, g], low[:, g] = np.where(bad, np.nan, s), np.where(bad, np.nan, mn)
    return codes, scale, low


def values(codes, scale, low, group):
    """The weights in 64 bits."""
    K = codes.shape[1]
    at = np.arange(K) // group
    return low.astype(np.float64)[:, at] + codes * scale.astype(np.float64)[:, at]


def pack(codes, scale, low, group):
    """The documented layout, a code at a time."""
    N, K = codes.shape
    rows, blocks = -(-N // 16), -(-K // 128)
    groups = blocks * 128 // group
    words = np.zeros((rows, blocks, 64, 4), np.uint32)
    n, k = np.meshgrid(np.arange(N), np.arange(K), indexing="ij")
    c = k % 8
    np.bitwise_or.at(words, (n // 16, k // 128, n % 16 + 16 * (k % 32 // 8), k % 128 // 32), codes.astype(np.uint32) << (4 * (c // 2 + 4 * (c % 2))).astype(np.uint32))
    levels = np.zeros((rows, groups, 16), np.uint32)
    top = lambda x: x.astype(np.float32).view(np.uint32) >> 16  # noqa: E731
    for g in range(scale.shape[1]):
        levels[np.arange(N) // 16, g, np.arange(N) % 16] = top(scale[:, g].copy()) | top(low[:, g].copy()) << 16
    return np.concatenate([words.reshape(-1).view(np.uint8), levels.reshape(-1).view(np.uint8)])


# ------------------------------------------------------------------ routing

def scores_of(x, score):
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        if score == "sigmoid":
            return 1 / (1 + np.exp(-x))
        e = np.exp(x - x.max(-1, keepdims=True))
        return np.where((x == -np.inf).all(-1, keepdims=True), 0.0, e / e.sum(-1, keepdims=True))     # of nothing


def route(x, k, score="softmax", bias=None, groups=1, top_groups=1, group_score="best", renormalise=True, scale=1.0):
    """ids [T, k] and weights in 64 bits, a token at a time."""
    x = np.asarray(x, np.float64)
    T, E = x.shape
    s = scores_of(x, score)
    ids, weights = np.full((T, k), -1), np.zeros((T, k))
    for t in range(T):
        rank = (s[t] + np.asarray(bias, np.float64) if bias is not None else x[t]).copy()
        worth = (s[t] + (np.asarray(bias, np.float64) if bias is not None else 0)) if group_score == "two" else rank.copy()
        out = ~(x[t] > -np.inf) | ~(rank > -np.inf)
        rank[out] = -np.inf
        if groups > 1:
            per, best = E // groups, []
            for g in range(groups):
                had = sorted((w for w, o in zip(worth[g * per:(g + 1) * per], out[g * per:(g + 1) * per]) if not o), reverse=True)
                best.append(-np.inf if not had else sum(had[:2]) if group_score == "two" else had[0])
            kept = sorted(range(groups), key=lambda g: (-best[g], g))[:top_groups]
            for g in range(groups):
                if g not in kept or best[g] == -np.inf:
                    rank[g * per:(g + 1) * per] = -np.inf
        order = [e for e in sorted(range(E), key=lambda e: (-rank[e], e)) if rank[e] > -np.inf][:k]
        ids[t, :len(order)] = order
        picked = s[t, order]
        if renormalise:
            picked = picked / picked.sum() if len(order) and picked.sum() > 0 else 0 * picked
        weights[t, :len(order)] = scale * picked
        if np.isnan(x[t]).any() or (score == "softmax" and (x[t] == np.inf).any()):
            weights[t] = np.nan
    return ids, weights


def route_gradient(x, ids, g, score="softmax", renormalise=True, scale=1.0):
    """Of sum(g * weights) in the logits, by the Jacobian of scores and shares."""
    x, g = np.asarray(x, np.float64), np.asarray(g, np.float64)
    T, E = x.shape
    s = scores_of(x, score)
    out = np.zeros((T, E))
    for t in range(T):
        e = ids[t][ids[t] >= 0]
        gt = scale * g[t][ids[t] >= 0]
        p = s[t, e]
        if renormalise:
            S = p.sum()
            if not S > 0:
                continue
            gt = gt / S - (gt * p).sum() / S ** 2
        of_scores = np.zeros(E)
        of_scores[e] = gt
        if score == "softmax":
            out[t] = (np.diag(s[t]) - np.outer(s[t], s[t])) @ of_scores
        else:
            out[t] = of_scores * s[t] * (1 - s[t])
    return out


# ------------------------------------------------------------------ turned rows

def turn(x, positions, frequencies, interleaved=False, scale=1.0):
    """[T, heads, d] in 64 bits."""
    x = np.asarray(x, np.float64).copy()
    P = len(frequencies)
    i = np.arange(P)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + P)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(frequencies, np.float64)
    z = (x[..., a] + 1j * x[..., b]) * (scale * np.exp(1j * angle))[:, None, :]
    x[..., a], x[..., b] = z.real, z.imag
    return x
