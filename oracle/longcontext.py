"""Rotary positions, bounds of pages and attention over a choice of pages, in 64 bits (test infrastructure, CPU only).

Rotation: pair i of the `dims` leading elements of a head turns by position * f_i, f_i = base^(-2i/dims), divided by `factor` or,
with an original length, by parts: pairs that turn often over that length keep f_i, those that hardly turn get f_i / factor.
Choice: with more than `budget` pages visible, the first `first`, the last `last` and those of the highest score between;
a page's score is what the sum of the group's logits with any key inside the page's bounds does not exceed.
"""
import math

import numpy as np


def frequencies(dims, base=10000.0, factor=1.0, original_len=0, low_turns=1.0, high_turns=32.0):
    out = []
    for i in range(dims // 2):
        f = base ** (-2.0 * i / dims)
        if original_len:
            turns = original_len * f / (2 * math.pi)
            keep = min(max((turns - low_turns) / (high_turns - low_turns), 0.0), 1.0)
            f = keep * f + (1 - keep) * f / factor
        else:
            f = f / factor
        out.append(f)
    return np.array(out)


def turn(x, positions, freq, layout="halves", magnitude=1.0):
    """x [n, heads, D] at positions [n]; float64, not rounded."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    half = len(freq)
    angle = np.asarray(positions, np.float64)[:, None] * freq            # [n, pairs]
    c, s = magnitude * np.cos(angle)[:, None], magnitude * np.sin(angle)[:, None]
    a, b = (slice(0, half), slice(half, 2 * half)) if layout == "halves" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def page_bounds(K):
    """K [tokens, Hkv, D] -> [full pages, Hkv, 2, D]."""
    full = len(K) // 16
    pages = np.asarray(K)[:full * 16].reshape(full, 16, *K.shape[1:])
    return np.stack([pages.min(1), pages.max(1)], 2)


def scores(q, bounds):
    """q [G, D] of one kv head, bounds [pages, 2, D] -> [pages], rounded to 32 bits."""
    q, b = np.asarray(q, np.float64), np.asarray(bounds, np.float64)
    with np.errstate(invalid="ignore"):
        up, down = np.where(q < 0, 0, q).sum(0), np.where(q > 0, 0, q).sum(0)
        return ((up * b[:, 1]).sum(-1) + (down * b[:, 0]).sum(-1)).astype(np.float32)


def choose(score_of, n, budget, first, last):
    """Indices of the pages read, ascending; score_of[p] for p in [first, n - last)."""
    if n <= budget:
        return list(range(n))
    between = range(first, n - last)
    rank = sorted(between, key=lambda p: (0 if np.isnan(score_of[p]) else 1, 0.0 if np.isnan(score_of[p]) else -float(score_of[p]), p))
    return sorted(list(range(first)) + rank[:budget - first - last] + list(range(n - last, n)))


def sparse_attention(q, K, V, len_before, budget, first, last, scale=None):
    """q [n, Hq, D] (as stored), K, V [len_before + n, Hkv, D] (as stored) -> out [n, Hq, D] float64, pages [n][Hkv] lists."""
    n, Hq, D = q.shape
    Hkv = K.shape[1]
    G = Hq // Hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, picked = np.zeros((n, Hq, D)), []
    bounds = page_bounds(K)
    for i in range(n):
        seen = len_before + i + 1
        count = -(-seen // 16)
        picked.append([])
        for g in range(Hkv):
            qg = np.asarray(q[i, g * G:(g + 1) * G], np.float64)
            sc = scores(qg, bounds[:count, g]) if count > budget else None
            pages = choose(sc, count, budget, first, last)
            at = np.concatenate([np.arange(16 * p, min(16 * p + 16, seen)) for p in pages])
            s = qg @ np.asarray(K[at, g], np.float64).T * scale
            w = np.exp(s - s.max(1, keepdims=True))
            out[i, g * G:(g + 1) * G] = (w / w.sum(1, keepdims=True)) @ np.asarray(V[at, g], np.float64)
            picked[-1].append(pages)
    return out, picked
