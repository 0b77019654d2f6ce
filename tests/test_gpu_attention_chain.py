"""Trees that are chains, on the GPU: what `attend` computes for them, bit for bit where both run the same kernel on the same tiles."""
import numpy as np
import pytest
import torch

import tree_helpers as th
import tree_oracle
from paper_2411_19379_amd import attention as attn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# Without a window tiles of keys begin at the same keys, and either up to 32 rows per key head, more than 256, or fp32.
@pytest.mark.parametrize("hq,hkv,d,bs,dtype,new,cached", [
    (4, 1, 128, 16, "bf16", [8, 1, 0, 5], [40, 0, 77, 2000]), (8, 2, 64, 4, "f16", [3], [700]), (12, 12, 64, 16, "bf16", [1] * 40, list(range(0, 400, 10))),
    (8, 2, 64, 16, "bf16", [100, 5, 1], [100, 31, 64]), (8, 1, 128, 32, "f16", [60], [3000]), (4, 2, 64, 16, "f32", [40, 5, 1], [100, 31, 640]),
    (3, 1, 128, 8, "f32", [1], [900])])
def test_a_chain_is_attend(hq, hkv, d, bs, dtype, new, cached):
    p = th.make(3, hq, hkv, d, bs, dtype, new, cached, max_new=max(new))
    positions, seen = tree_oracle.draft_tree(np.concatenate([np.arange(n) - 1 for n in new]), p.cu, p.cached, p.words)
    ints = lambda v: torch.as_tensor(np.asarray(v), dtype=torch.int32, device=DEV)
    layer = p.q.to(DEV), p.k_cache.to(DEV), p.v_cache.to(DEV), ints(p.table), ints(p.cu), ints(p.cached)
    kw = dict(scale=p.scale, max_new=p.max_new, return_lse=True)
    want, got = attn.attend(*layer, **kw), attn.attend_tree(*layer, ints(positions), ints(tree_oracle.bits_of(seen, p.words)), **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
