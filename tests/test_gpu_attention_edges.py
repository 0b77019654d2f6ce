"""The attention operators on the GPU where a caller's arrays end early or values are extreme."""
import numpy as np
import pytest
import torch

from test_attention_malformed import NARROW, narrow_problem

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", sorted(NARROW))
def test_assign_with_a_table_that_is_too_narrow(name, in_place):
    """No block is lost behind the end of a row, and `counts` says how many were missing there."""
    from paper_2411_19379_amd import attention as attn
    print(f"assign narrow {name}", flush=True)
    (bs, T, cu, cached, table, free, n_free, shared), want = narrow_problem(name)
    step = attn.assign_blocks(bs, T, _dev(cu), _dev(cached), _dev(table), _dev(free), _dev(np.array([n_free], np.int32)),
                              shared_tail=_dev(shared), in_place=in_place)
    for g, w, what in zip(step, want, ("table", "slots", "positions", "copies", "counts")):
        assert np.array_equal(g.cpu().numpy(), w), f"{name}: {what}"
