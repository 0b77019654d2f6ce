"""Steps that check trees of drafted tokens from their definitions, in plain Python and 64 bits: one request and one token after
the other.  Nothing here knows words of bits, tiles or splits."""
from __future__ import annotations

import math

import numpy as np


def branch(parents, i):
    """A token and its ancestors, itself first."""
    line = []
    while i >= 0:
        line.append(i)
        i = parents[i] if 0 <= parents[i] < i else -1
    return line


def draft_tree(parents, cu, cached, words, window=0, sinks=0):
    """Positions [T] and, for every token, the set of new tokens of its sequence that it sees."""
    T = len(parents)
    positions, seen = np.zeros(T, np.int32), [set() for _ in range(T)]
    for b in range(len(cached)):
        start, n = int(cu[b]), int(cu[b + 1]) - int(cu[b])
        for i in range(n):
            if i >= 32 * words:
                positions[start + i] = cached[b]
                continue
            line = branch(parents[start:start + n], i)
            depth = {a: len(line) - 1 - k for k, a in enumerate(line)}
            positions[start + i] = cached[b] + depth[i]
            seen[start + i] = {a for a in line if window == 0 or depth[i] - depth[a] < window or cached[b] + depth[a] < sinks}
    return positions, seen


def bits_of(seen, words):
    out = np.zeros((len(seen), words), np.uint32)
    for t, s in enumerate(seen):
        for j in s:
            if j < 32 * words:
                out[t, j // 32] |= np.uint32(1 << (j % 32))
    return out.view(np.int32)


def attend_tree(q, k_cache, v_cache, table, cu, cached, positions, seen, scale, window=0, sinks=0):
    """As `attn_oracle.attend`; `seen`: sets of new tokens."""
    T, hq, d = q.shape
    n_blocks, hkv, bs, _ = k_cache.shape
    out, lse = np.zeros((T, hq, d)), np.full((T, hq), -np.inf)
    with np.errstate(all="ignore"):
        for b in range(len(cached)):
            c = int(cached[b])
            for i in range(int(cu[b + 1]) - int(cu[b])):
                t = int(cu[b]) + i
                p = min(max(int(positions[t]), c), c + i)
                keys = [j for j in range(c) if window == 0 or j > p - window or j < sinks] + [c + j for j in sorted(seen[t]) if j <= i]
                keys = [j for j in keys if j // bs < table.shape[1] and 0 <= table[b, j // bs] < n_blocks]
                if not keys:
                    continue
                blocks, rows = table[b, np.array(keys) // bs], np.array(keys) % bs
                for h in range(hq):
                    g = h // (hq // hkv)
                    k, v = k_cache[blocks, g, rows], v_cache[blocks, g, rows]
                    s = (k @ q[t, h]) * scale
                    top = s.max() if not np.isnan(s).any() else np.nan
                    w = np.exp(s - top)
                    out[t, h] = (w[:, None] * v).sum(0) / w.sum()
                    lse[t, h] = top + math.log(w.sum()) if w.sum() > 0 else np.nan
    return out, lse


def accept_path(tokens, parents, choices, cu, cached, table=None, block_size=0, free=None, n_free=0):
    """path, counts, next tokens, kept lengths, the free list and its length."""
    T = len(tokens)
    path = np.full(T, -1, np.int32)
    counts, following, lens = [], [], []
    free, left = (list(map(int, free)) if free is not None else None), min(max(int(n_free), 0), len(free) if free is not None else 0)
    for b in range(len(cached)):
        start, n, c = int(cu[b]), int(cu[b + 1]) - int(cu[b]), int(cached[b])
        kept = [0] if n else []
        while kept:
            v = kept[-1]
            more = [i for i in range(v + 1, n) if parents[start + i] == v and tokens[start + i] == choices[start + v]]
            if not more:
                break
            kept.append(more[0])
        path[start:start + len(kept)] = kept
        counts.append(len(kept))
        following.append(int(choices[start + kept[-1]]) if kept else -1)
        lens.append(c + len(kept))
        if table is not None:
            for e in range(-(-lens[-1] // block_size), min(-(-(c + n) // block_size), table.shape[1])):
                if table[b, e] >= 0 and left < len(free):
                    free[left] = int(table[b, e])
                    left += 1
    return path, np.array(counts, np.int32), np.array(following, np.int32), np.array(lens, np.int32), free, left


def keep_path(caches, table, cu, cached, path):
    """New caches [n_blocks, heads, block_size, d] with the kept rows in their places."""
    out = [np.array(c) for c in caches]
    n_blocks, _, bs, _ = out[0].shape

    def at(b, j):
        if j // bs >= table.shape[1] or not 0 <= table[b, j // bs] < n_blocks:
            return None
        return int(table[b, j // bs]), j % bs

    for b in range(len(cached)):
        start, n, c = int(cu[b]), int(cu[b + 1]) - int(cu[b]), int(cached[b])
        for k in range(n):
            i = int(path[start + k])
            if not k <= i < n:
                break
            source, target = at(b, c + i), at(b, c + k)
            if source is None or target is None or source == target:
                continue
            for cache in out:
                cache[target[0], :, target[1]] = cache[source[0], :, source[1]]
    return out


def random_parents(rng, n, chain=0.5, roots=0.0):
    """Token 0 a root; the others go on where the one in front is, start a branch, or (`roots`) a tree of their own."""
    parents = [-1] * n
    for i in range(1, n):
        u = rng.random()
        parents[i] = -1 if u < roots else i - 1 if rng.random() < chain else rng.randrange(i)
    return parents
