"""Oracle of the decode-step operators: plain, slow, numpy in 64 bits, from their formulas.

Inputs are numpy arrays (bf16 values widened to float64 by the caller). Where a test needs to know
how far a correct fp32 computation may be from the exact value, the function also returns the sum
of magnitudes that its rounding errors are relative to.
"""

import math

import numpy as np

ONE = 1 << 44


def _pairs(rotary, interleaved):
    i = np.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def _turn(x, positions, turns, interleaved, magnitude, sign=1.0):
    """Rows x [tokens, heads, dim] with each pair turned by the position's angle."""
    y = x.copy()
    if len(turns):
        a, b = _pairs(2 * len(turns), interleaved)
        part = np.outer(positions.astype(np.float64), turns)
        angle = 2 * math.pi * (part - np.rint(part))
        c, s = magnitude * np.cos(angle)[:, None], sign * magnitude * np.sin(angle)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def _spread(x, turns, interleaved, magnitude):
    """Magnitudes that feed each element of a turned row."""
    m = np.abs(x)
    if len(turns):
        a, b = _pairs(2 * len(turns), interleaved)
        both = abs(magnitude) * (m[..., a] + m[..., b])
        m[..., a], m[..., b] = both, both
    return m


def norm_rotate(x, gamma, positions, turns, interleaved=False, magnitude=1.0, eps=1e-6):
    """(rows, magnitudes): rows x normed (with a gamma) and turned; padding tokens are zeros."""
    live = (positions >= 0)[:, None, None]
    n = np.where(live, x, 0.0)
    if gamma is not None:
        n = n / np.sqrt(np.where(live, np.mean(n * n, -1, keepdims=True) + eps, 1.0)) * gamma
    return (np.where(live, _turn(n, positions, turns, interleaved, magnitude), 0.0),
            np.where(live, _spread(n, turns, interleaved, magnitude), 0.0))


def norm_rotate_back(dy, x, gamma, positions, turns, interleaved=False, magnitude=1.0, eps=1e-6):
    """(dx, its magnitudes, dgamma, its magnitudes); the latter two None without a gamma."""
    live = (positions >= 0)[:, None, None]
    dy = np.where(live, dy, 0.0)
    d = np.where(live, _turn(dy, positions, turns, interleaved, magnitude, -1.0), 0.0)
    dm = _spread(dy, turns, interleaved, magnitude)
    if gamma is None:
        return d, dm, None, None
    x = np.where(live, x, 0.0)
    r = 1.0 / np.sqrt(np.where(live, np.mean(x * x, -1, keepdims=True) + eps, 1.0))
    dx = r * (d * gamma - x * r * r * np.mean(d * gamma * x, -1, keepdims=True))
    mag = r * (dm * np.abs(gamma) + np.abs(x) * r * r * np.mean(dm * np.abs(gamma * x), -1, keepdims=True))
    return np.where(live, dx, 0.0), mag, (d * x * r).sum((0, 1)), (dm * np.abs(x) * r).sum((0, 1))


def attend(q, k_cache, v_cache, table, lengths, scale):
    """(out, lse, weighted magnitudes of the values, largest sum of magnitudes behind a score) of q
    [sequences, heads, dim] over caches [pages, heads, page_tokens, dim]."""
    n, hq, dim = q.shape
    pages, hk, page, _ = k_cache.shape
    out, mag = np.zeros((n, hq, dim)), np.zeros((n, hq, dim))
    lse, big = np.full((n, hq), -np.inf), np.zeros((n, hq))
    for s in range(n):
        tokens = [(int(table[s, j // page]), j % page) for j in range(min(max(int(lengths[s]), 0), table.shape[1] * page))]
        tokens = [(p, r) for p, r in tokens if 0 <= p < pages]
        if not tokens:
            continue
        p, r = (np.array(t) for t in zip(*tokens))
        for h in range(hq):
            k, v = k_cache[p, h // (hq // hk), r], v_cache[p, h // (hq // hk), r]
            x = scale * (k @ q[s, h])
            top = x.max()
            e = np.exp(x - top)
            w = e / e.sum()
            out[s, h], mag[s, h] = w @ v, w @ np.abs(v)
            lse[s, h] = top + math.log(e.sum())
            big[s, h] = abs(scale) * (np.abs(k) @ np.abs(q[s, h])).max()
    return out, lse, mag, big


def draw(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, most=float(np.finfo(np.float32).max)):
    """(token, log probability) of one row of logits (float32 values), in whole numbers of any size. most: the largest finite
    number of the logits' type, which +inf counts as."""
    l = np.minimum(np.where(np.isnan(logits), -np.inf, logits.astype(np.float64)), most)
    top = l.max()
    if top == -np.inf:
        return -1, -math.inf
    if not temperature > 0:
        return int(np.argmax(l)), 0.0
    live = l > -np.inf  # whatever the temperature
    w = np.zeros(len(l), np.int64)
    w[live] = np.rint(np.exp((l[live] - top) * (1.0 / float(np.float32(temperature)))) * ONE).astype(np.int64)
    w = w.tolist()
    order = np.argsort(-l, kind="stable").tolist()
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        parts = int(np.rint(max(float(np.float32(top_p)), 0.0) * 2 ** 24))
        need, total, kept = (sum(w[i] for i in order) * parts) >> 24, 0, []
        for i in order:
            if kept and total >= need:
                break
            kept.append(i)
            total += w[i]
        order = kept
    least = int(np.rint(min(max(float(np.float32(min_p)), 0.0), 1.0) * ONE))
    kept = sorted(i for i in order if w[i] >= least)
    total = sum(w[i] for i in kept)
    u = float(np.float32(u))
    at = (total * (0 if not u > 0 else min(int(u * 2 ** 24), 2 ** 24 - 1))) >> 24
    for i in kept:
        if at < w[i]:
            return i, math.log(w[i] / total)
        at -= w[i]
    raise AssertionError("the drawn share lies inside the kept weight")
