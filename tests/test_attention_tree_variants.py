"""The kernel of drafted trees in all its forms (two and four waves, one or two tiles of rows, heads of 64 and 128, keys of a wave in one
block or in several) against the definition in 64 bits, on the emulator and on the GPU: random bits with empty rows among them, missing
blocks, windows, more rows than the caller has said, infinities and NaN."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import attn_helpers as ah
import test_attention_tree_emulation as emulation
import tree_helpers as th
from paper_2411_19379_amd import attention as attn
from test_attention_tree_emulation import emu  # noqa: F401 (a fixture)

DEV = "cuda:0"

# heads, key heads, head_dim, block size, type, new tokens, cached tokens, window, sinks, max_new
CASES = {}
for _dtype in ("bf16", "f16"):
    for _d in (64, 128):
        # 33 to 64 rows per key head: two waves, 16 keys each
        CASES[f"two_{_dtype}_{_d}"] = (4, 1, _d, 16, _dtype, [11, 3, 0, 16], [70, 0, 5, 33], 0, 0, 16)
        CASES[f"two_blocks_{_dtype}_{_d}"] = (3, 1, _d, 4, _dtype, [13, 20], [40, 65], 0, 0, 20)
        # 65 to 128: four, 8 keys each
        CASES[f"four_{_dtype}_{_d}"] = (4, 2, _d, 8, _dtype, [50, 7, 1], [33, 90, 0], 0, 0, 50)
        CASES[f"four_blocks_{_dtype}_{_d}"] = (5, 1, _d, 2, _dtype, [25, 9], [31, 70], 0, 0, 25)
CASES.update({
    "two_window": (4, 2, 64, 16, "bf16", [30, 20], [150, 40], 5, 3, 30),
    "two_blocks_window": (2, 1, 128, 1, "f16", [25, 32], [97, 10], 40, 20, 32),
    "four_window": (2, 1, 128, 32, "f16", [60, 33], [120, 64], 9, 70, 60),
    "four_blocks_window": (6, 2, 64, 4, "bf16", [40, 1], [99, 200], 33, 2, 40),
    "two_and_more_rows": (4, 1, 64, 8, "bf16", [90, 2], [40, 30], 0, 0, 10),
    "four_and_more_rows": (2, 1, 128, 16, "f16", [130, 5], [7, 64], 0, 0, 40),
    "four_and_more_rows_window": (2, 1, 64, 4, "bf16", [150], [80], 12, 5, 50),
    # more than 128 rows, and 256 sequences and key heads: two tiles of four waves
    "two_tiles": (192, 64, 64, 16, "bf16", [70, 50, 1, 3], [60, 0, 33, 5], 0, 0, 70),
})
# where the rows of a tile are cut into splits by few and by many workgroups
ON_GPU = dict(CASES)
ON_GPU.update({
    "two_long": (8, 2, 128, 16, "bf16", [16, 9], [3000, 700], 0, 0, 16),
    "two_blocks_long": (8, 2, 64, 8, "f16", [12] * 20, [100 * k for k in range(20)], 0, 0, 12),
    "four_long": (32, 8, 128, 16, "f16", [32, 20, 5], [4000, 1234, 0], 0, 0, 32),
    "four_blocks_long": (8, 1, 128, 4, "bf16", [16, 10], [2000, 50], 0, 0, 16),
    "two_tiles_long": (32, 8, 128, 16, "bf16", [64, 40] + [1, 0, 5] * 10, [2000, 700] + [20 * k for k in range(30)], 0, 0, 64),
    "two_tiles_window": (32, 8, 64, 4, "f16", [50, 64] + [3, 1, 9] * 10, [500, 1200] + [30 * k for k in range(30)], 100, 4, 64),
})


def _not_finite(p):
    """Infinities and NaN in some values of K and V, of cached and new tokens, and in rows that hold no key."""
    rng = np.random.RandomState(5)
    for cache in (p.k_cache, p.v_cache):
        for bad in (float("inf"), float("nan"), -float("inf")):
            cache[rng.randint(cache.shape[0]), rng.randint(p.hkv), rng.randint(p.bs), rng.randint(p.d)] = bad


def _problem(case, bits, holes=0.0, not_finite=False):
    p = th.make(41, *case, bits=bits, holes=holes)
    if not_finite:
        _not_finite(p)
    return p


KINDS = {"tree": dict(bits="tree"), "any": dict(bits="any"), "holes": dict(bits="any", holes=0.1), "not_finite": dict(bits="any", not_finite=True)}


# each kind in its turn, half of them with copies into LDS as late as their wait allows, few workgroups or many
@pytest.mark.parametrize("at,name", list(enumerate(sorted(set(CASES) - {"two_tiles"}))))
def test_emulated(emu, tmp_path, at, name):  # noqa: F811
    p = _problem(CASES[name], **KINDS[sorted(KINDS)[at % 4]])
    out, lse = emulation._attend(emu, tmp_path, p, *((0, "end", 60, 0) if at % 3 else (5, "start", 2, 1)))
    ah.check(p, out, lse, name, th.reference(p))


def test_two_tiles_emulated(emu, tmp_path):  # noqa: F811
    p = _problem(CASES["two_tiles"], "tree")
    ah.check(p, *emulation._attend(emu, tmp_path, p, 1, "end", 300, 1), "two_tiles", th.reference(p))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("name", sorted(ON_GPU))
def test_on_the_gpu(name, kind):
    p = _problem(ON_GPU[name], **KINDS[kind])
    ints = lambda v: torch.as_tensor(np.asarray(v), dtype=torch.int32, device=DEV)
    args = (p.q.to(DEV), p.k_cache.to(DEV), p.v_cache.to(DEV), ints(p.table), ints(p.cu), ints(p.cached), ints(p.positions), ints(p.bits))
    ref = th.reference(p)
    for max_new in (p.max_new, 0):  # a hint picks a kernel, and nothing else
        out, lse = attn.attend_tree(*args, scale=p.scale, window=p.window, sinks=p.sinks, max_new=max_new, return_lse=True)
        ah.check(p, out.cpu().double().numpy(), lse.cpu().numpy(), name, ref)
