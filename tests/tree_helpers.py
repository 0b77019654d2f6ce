"""Problems for the operators of steps with trees, shared by the emulation and the GPU tests."""
from __future__ import annotations

import random

import numpy as np

import attn_helpers as ah
import tree_oracle


def make(seed, hq, hkv, d, bs, dtype, new, cached, window=0, sinks=0, max_new=0, chain=0.5, bits="tree", **more):
    """An attention problem whose new tokens are trees.  `bits`: those of the trees, or random ones with empty rows among them."""
    p = ah.make(seed, hq, hkv, d, bs, dtype, new, cached, window, sinks, max_new, **more)
    rng = random.Random(seed)
    p.words = max(1, (max(list(new) + [1]) + 31) // 32)
    p.parents = np.array([x for n in new for x in tree_oracle.random_parents(rng, n, chain, 0.1)], np.int32)
    p.positions, p.seen = tree_oracle.draft_tree(p.parents, p.cu, p.cached, p.words, window, sinks)
    if bits == "any":
        for b, n in enumerate(new):
            for i in range(n):
                t = int(p.cu[b]) + i
                # bits behind the token's own count for nothing
                p.seen[t] = {j for j in range(n) if rng.random() < 0.3} if rng.random() < 0.7 else set()
                p.positions[t] = cached[b] + rng.randrange(-3, i + 4)
    p.bits = tree_oracle.bits_of(p.seen, p.words)
    return p


def reference(p):
    q, k, v = (x.double().numpy() for x in (p.q, p.k_cache, p.v_cache))
    args = p.table, p.cu, p.cached, p.positions, p.seen, p.scale, p.window, p.sinks
    out, lse = tree_oracle.attend_tree(q, k, v, *args)
    size, _ = tree_oracle.attend_tree(q, k, np.abs(v), *args)
    return out, lse, size


def accept_problem(seed, batch, most, bs, width=None, vocabulary=3, holes=0.0):
    rng = random.Random(seed)
    new = [rng.choice([0, 1, rng.randrange(1, most + 1), rng.randrange(1, most + 1)]) for _ in range(batch)]
    cached = [rng.randrange(0, 5 * bs) for _ in range(batch)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    parents = np.array([x for n in new for x in tree_oracle.random_parents(rng, n, 0.6, 0.05)], np.int32)
    T = int(cu[-1])
    tokens, choices = (np.array([rng.randrange(vocabulary) for _ in range(T)], np.int32) for _ in range(2))
    blocks = [-(-(c + n) // bs) for c, n in zip(cached, new)]
    table = np.full((batch, width or max(blocks + [1])), -1, np.int32)
    at = 0
    for b, n in enumerate(blocks):
        n = min(n, table.shape[1])
        table[b, :n] = range(at, at + n)
        at += n
    if holes:
        table[np.random.RandomState(seed).rand(*table.shape) < holes] = -1
    return dict(new=new, cached=np.array(cached, np.int32), cu=cu, parents=parents, tokens=tokens, choices=choices, table=table, T=T,
                n_blocks=max(at, 1))


# heads, key heads, head_dim, block size, type, new tokens, cached tokens, window, sinks, max_new
CASES = {
    "one_token": (4, 1, 128, 16, "bf16", [1], [0], 0, 0, 1),
    "one_each": (8, 2, 64, 8, "f16", [1, 1, 0, 1], [37, 200, 9, 63], 0, 0, 1),
    "few": (4, 2, 128, 16, "f16", [5, 2, 1, 7], [40, 0, 77, 30], 0, 0, 7),
    "few_wide": (12, 1, 64, 16, "bf16", [2], [61], 0, 0, 2),
    "few_window": (3, 3, 64, 4, "bf16", [1, 10], [150, 97], 6, 3, 10),
    "few_by_a_wrong_hint": (2, 1, 64, 16, "f16", [40, 3], [5, 30], 0, 0, 1),
    "chunk": (2, 2, 64, 16, "bf16", [70], [33], 0, 0, 0),
    "chunk_group": (4, 1, 128, 16, "f16", [67, 1, 0, 20], [10, 80, 5, 0], 0, 0, 0),
    "chunk_group3": (3, 1, 64, 1, "bf16", [100], [0], 0, 0, 0),
    "chunk_window": (2, 1, 64, 32, "bf16", [150], [100], 7, 5, 0),
    "chunk_window_sinks_reach_new": (2, 2, 64, 16, "f16", [65, 3], [20, 64], 3, 24, 0),
    "chunk_one_sequence_of_many": (4, 2, 64, 16, "bf16", [1, 1, 1, 40, 1], [140, 63, 64, 65, 0], 0, 0, 40),
    "f32": (4, 2, 64, 16, "f32", [37, 1], [20, 64], 0, 0, 0),
    "f32_window": (2, 1, 128, 8, "f32", [40, 0, 2], [61, 7, 33], 17, 2, 0),
}
