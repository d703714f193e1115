"""Oracle of the operators for several new tokens of a sequence: plain, slow, numpy in 64 bits, from their definitions."""

import math

import numpy as np


def spans(starts, tokens):
    """(first row, number) of each sequence's new tokens; entries outside count as the nearest."""
    at = [min(max(int(s), 0), tokens) for s in starts]
    return [(a, max(b - a, 0)) for a, b in zip(at, at[1:])]


def branch(parents, i):
    """The new tokens from i back to the cached ones; parents None: a chain."""
    got = [i]
    while True:
        p = i - 1 if parents is None else int(parents[i])
        if not 0 <= p < i:
            return got
        got.append(p)
        i = p


def lay(starts, lengths, tokens, parents=None, words=0):
    """(seq_of, positions, places, seen), masks as rows of 64-bit words (None without words)."""
    seq_of, positions, places = (np.full(tokens, -1, np.int32) for _ in range(3))
    seen = np.zeros((tokens, words), np.uint64)
    for s, (first, count) in enumerate(spans(starts, tokens)):
        own = None if parents is None else parents[first:first + count]
        cached = max(int(lengths[s]), 0)
        for i in range(count):
            if words and i >= 64 * words:
                continue
            seq_of[first + i] = s
            places[first + i] = min(cached + i, 2 ** 31 - 1)
            if parents is None and words == 0:
                positions[first + i] = places[first + i]
                continue
            on = branch(own, i)
            positions[first + i] = min(cached + len(on) - 1, 2 ** 31 - 1)
            for j in on:
                seen[first + i, j // 64] |= np.uint64(1 << (j % 64))
    return seq_of, positions, places, seen.view(np.int64) if words else None


def attend(q, k_cache, v_cache, table, lengths, starts, seen, scale):
    """(out, lse, weighted magnitudes of the values, largest sum of magnitudes behind a score) of q [tokens, heads, dim] over caches
    [pages, heads, page_tokens, dim]; seen: rows of 64-bit words, or None. Rows of no sequence: NaN."""
    n, hq, dim = q.shape
    pages, hk, page, _ = k_cache.shape
    out, mag = np.full((n, hq, dim), np.nan), np.zeros((n, hq, dim))
    lse, big = np.full((n, hq), np.nan), np.zeros((n, hq))
    room = table.shape[1] * page
    for s, (first, count) in enumerate(spans(starts, n)):
        cached = max(int(lengths[s]), 0)
        places = [(j, int(table[s, j // page]), j % page) for j in range(min(cached + count, room))]
        places = [p for p in places if 0 <= p[1] < pages]
        j, p, r = (np.array(x, np.int64) for x in zip(*places)) if places else (np.zeros(0, np.int64),) * 3
        e = j - cached
        for i in range(count):
            if seen is None:
                live = e <= i
            else:
                words = seen[first + i].astype(np.int64).view(np.uint64)
                live = np.array([x < 0 or (x < 64 * len(words) and bool(int(words[x // 64]) >> int(x % 64) & 1)) for x in e], bool)
            t = first + i
            out[t], lse[t] = 0.0, -np.inf
            if not live.any():
                continue
            for h in range(hq):
                k, v = k_cache[p[live], h // (hq // hk), r[live]], v_cache[p[live], h // (hq // hk), r[live]]
                x = scale * (k @ q[t, h])
                top = x.max()
                w = np.exp(x - top)
                total = w.sum()
                out[t, h], mag[t, h] = (w / total) @ v, (w / total) @ np.abs(v)
                lse[t, h] = top + math.log(total)
                big[t, h] = abs(scale) * (np.abs(k) @ np.abs(q[t, h])).max()
    return out, lse, mag, big


def accept(drafted, drawn, starts, most, parents=None, words=0):
    """(path, tokens, counts) of the walk along the drafted tokens that the draws agree with, among the first 64 words of a tree."""
    at = spans(starts, len(drafted))
    path, won, counts = np.full((len(at), most), -1, np.int32), np.full((len(at), most), -1, np.int32), np.zeros(len(at), np.int32)
    for s, (first, count) in enumerate(at):
        count = min(count, 64 * words) if words else count
        i = 0 if count else None
        while i is not None and counts[s] < most:
            path[s, counts[s]], won[s, counts[s]] = i, drawn[first + i]
            counts[s] += 1
            behind = [j for j in range(i + 1, count) if (j - 1 if parents is None else parents[first + j]) == i]
            i = next((j for j in behind if drafted[first + j] == drawn[first + i] >= 0), None)
    return path, won, counts


def keep(cache, table, lengths, path):
    """The cache [pages, heads, page_tokens, dim] with each sequence's path brought together (a copy)."""
    got = cache.copy()
    pages, _, page, _ = cache.shape

    def place(s, j):
        if j // page < table.shape[1] and 0 <= table[s, j // page] < pages:
            return int(table[s, j // page]), j % page
        return None

    for s, row in enumerate(path):
        cached, before = max(int(lengths[s]), 0), -1
        for i, p in enumerate(row):
            if p < 0 or p <= before:
                break
            before = p
            src, dst = place(s, cached + int(p)), place(s, cached + i)
            if src and dst:
                got[dst[0], :, dst[1]] = cache[src[0], :, src[1]]
    return got
