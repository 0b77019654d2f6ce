"""Problems for the attention operators and the bounds their results are held to, shared by the emulation and the GPU tests."""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np
import torch

import attn_oracle

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CODE = {"f32": 0, "bf16": 1, "f16": 2}


@dataclass
class Problem:
    hq: int
    hkv: int
    d: int
    bs: int
    dtype: str
    new: list
    cached: list
    window: int
    sinks: int
    max_new: int
    scale: float
    q: torch.Tensor
    k_cache: torch.Tensor
    v_cache: torch.Tensor
    table: np.ndarray
    cu: np.ndarray

    @property
    def T(self):
        return int(self.cu[-1])

    def block_row(self, seq, j):
        """Where the key at position j of a sequence lies in the caches."""
        return int(self.table[seq, j // self.bs]), j % self.bs


def make(seed, hq, hkv, d, bs, dtype, new, cached, window=0, sinks=0, max_new=0, spread=2.0, holes=0.0, spare=2):
    """Random inputs; the cache's unused rows hold NaN, `holes` of the table's entries name no block."""
    g = torch.Generator().manual_seed(seed)
    rs = np.random.RandomState(seed)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    blocks = [-(-(n + c) // bs) for n, c in zip(new, cached)]
    n_blocks = sum(blocks) + spare
    ids = rs.permutation(n_blocks)
    table = np.full((len(new), max(blocks + [1]) + 1), -1, np.int32)
    k = torch.full((n_blocks, hkv, bs, d), float("nan"))
    v = torch.full((n_blocks, hkv, bs, d), float("nan"))
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = ids[at:at + n]
        at += n
        for j in range(new[b] + cached[b]):
            k[table[b, j // bs], :, j % bs] = torch.randn((hkv, d), generator=g)
            v[table[b, j // bs], :, j % bs] = torch.randn((hkv, d), generator=g)
    if holes:
        # ids that name nothing: negative ones, and ones behind the cache's end
        out = rs.rand(*table.shape) < holes
        table = np.where(out & (table >= 0), rs.choice([-1, -7, n_blocks, 2 ** 31 - 1], size=table.shape), table).astype(np.int32)
    q = torch.randn((int(cu[-1]), hq, d), generator=g) * spread
    t = TORCH[dtype]
    return Problem(hq, hkv, d, bs, dtype, list(new), list(cached), window, sinks, max_new, d ** -0.5, q.to(t), k.to(t), v.to(t), table, cu)


def reference(p: Problem):
    """out, lse and the weighted mean of |v|, which the error of a weighted mean is proportional to."""
    q, k, v = (x.double().numpy() for x in (p.q, p.k_cache, p.v_cache))
    out, lse = attn_oracle.attend(q, k, v, p.table, p.cu, p.cached, p.scale, p.window, p.sinks)
    size, _ = attn_oracle.attend(q, k, np.abs(v), p.table, p.cu, p.cached, p.scale, p.window, p.sinks)
    return out, lse, size


def bounds(p: Problem, out, lse, size):
    """With u half an ulp of 1 in the storage type: the weights and the result are rounded once each, at most 2 u of the
    weighted mean of |v|; fp32 sums, products and powers of scores of at most some tens add 1e-5 of it.  Weights of fp16 below
    its smallest normal number are off by 2^-25 of the largest at most, and |v| is below 8."""
    u = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[p.dtype]
    keys = max([n + c for n, c in zip(p.new, p.cached)] + [1])
    tiny = keys * 8 * 2.0 ** -25 if p.dtype == "f16" else 1e-30
    return (2 * u + 1e-5) * size + tiny, 1e-5 * (1 + np.abs(lse))


def check(p: Problem, got, got_lse, what="", ref=None, sums=0.0):
    """`sums`: for scores beyond the tens that `bounds` covers, the largest scale * sum |q k| of the problem.  d / 4 rounded
    sums and two more roundings put a score off by that many half ulps of it, weight and sum of weights by as much each."""
    out, lse, size = ref or reference(p)
    tol, tol_lse = bounds(p, out, lse, size)
    off = (p.d / 4 + 2) * 2.0 ** -24 * sums
    tol, tol_lse = tol + 2 * off * size, tol_lse + off
    got, got_lse = np.asarray(got, np.float64), np.asarray(got_lse, np.float64)
    fine = np.isfinite(out)
    assert np.array_equal(np.isnan(got), np.isnan(out)), f"{what}: NaN in other places than the definition's"
    assert np.array_equal(got[~fine & ~np.isnan(out)], out[~fine & ~np.isnan(out)]), f"{what}: infinities differ"
    with np.errstate(invalid="ignore"):
        far = np.where(fine, np.abs(got - out) / tol, 0.0)
        worst = float(far.max()) if far.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times the bound at {np.unravel_index(far.argmax(), far.shape)}"
    fine = np.isfinite(lse)
    assert np.array_equal(got_lse[~fine], lse[~fine], equal_nan=True), f"{what}: lse of rows without a finite one differs"
    with np.errstate(invalid="ignore"):
        far = np.where(fine, np.abs(got_lse - lse) / tol_lse, 0.0)
    assert not far.size or far.max() <= 1.0, f"{what}: lse {far.max():.2f} times the bound"
    return worst
