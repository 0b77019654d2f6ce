"""The attention layers' operators from their definitions, in plain Python and 64 bits: one request after the other, one
token after the other, one key list per query.  Nothing here knows tiles, splits or running maxima."""
from __future__ import annotations

import math

import numpy as np


def assign(block_size, cu, cached, table, free, n_free, shared=None):
    """Returns table, slots, positions, copies, counts."""
    table = [list(map(int, r)) for r in table]
    width = len(table[0]) if table else 0
    left, missing = int(n_free), 0
    slots, positions, copies = [], [], []

    def take():
        nonlocal left, missing
        if left == 0:
            missing += 1
            return -1
        left -= 1
        return int(free[left])

    for b in range(len(cached)):
        n, c = int(cu[b + 1]) - int(cu[b]), int(cached[b])
        held = -(-c // block_size)
        copy = [-1, -1, 0, 0]
        if n and shared is not None and shared[b] and c % block_size:
            to = take()
            if held - 1 < width:
                copy = [table[b][held - 1], to, c % block_size, 0]
                table[b][held - 1] = to
        for e in range(held, width):
            table[b][e] = -1
        for p in range(c, c + n):
            e = p // block_size
            if e >= held:
                block = take()
                held += 1
                if e < width:
                    table[b][e] = block
            block = table[b][e] if e < width else -1
            slots.append(block * block_size + p % block_size if block >= 0 else -1)
            positions.append(p)
        copies.append(copy)
    return (np.array(table, np.int32).reshape(len(cached), width), np.array(slots, np.int64), np.array(positions, np.int32),
            np.array(copies, np.int32).reshape(-1, 4), np.array([left, missing], np.int32))


def turn(x, rows, rot, interleaved):
    """x [T, heads, d] float64, rows [T, 2, rot/2]: every pair as a complex number times its turn."""
    x = np.array(x, np.float64)
    if rot == 0:
        return x
    w = (rows[:, 0].astype(np.float64) + 1j * rows[:, 1].astype(np.float64))[:, None, :]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    z = (a + 1j * b) * w
    y = x.copy()
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def attend(q, k_cache, v_cache, table, cu, cached, scale, window=0, sinks=0):
    """q [T, hq, d], caches [n_blocks, hkv, bs, d] as float64; returns out [T, hq, d] and lse [T, hq]."""
    T, hq, d = q.shape
    n_blocks, hkv, bs, _ = k_cache.shape
    out, lse = np.zeros((T, hq, d)), np.full((T, hq), -np.inf)
    with np.errstate(all="ignore"):
        for b in range(len(cached)):
            for i in range(int(cu[b + 1]) - int(cu[b])):
                p = int(cached[b]) + i
                seen = [j for j in range(p + 1) if window == 0 or j > p - window or j < sinks]
                seen = [j for j in seen if j // bs < table.shape[1] and 0 <= table[b, j // bs] < n_blocks]
                if not seen:
                    continue
                blocks, rows = table[b, np.array(seen) // bs], np.array(seen) % bs
                for h in range(hq):
                    g = h // (hq // hkv)
                    k, v = k_cache[blocks, g, rows], v_cache[blocks, g, rows]
                    s = (k @ q[cu[b] + i, h]) * scale
                    top = s.max() if not np.isnan(s).any() else np.nan
                    w = np.exp(s - top)
                    # one product after the other: zero weights times infinities are NaN, as in the formula
                    out[cu[b] + i, h] = (w[:, None] * v).sum(0) / w.sum()
                    lse[cu[b] + i, h] = top + math.log(w.sum()) if w.sum() > 0 else np.nan
    return out, lse
