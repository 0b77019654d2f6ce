"""The attention operators on the GPU where a caller's arrays end early or values are extreme."""
import numpy as np
import pytest
import torch

import attn_helpers as ah
from test_attention_emulation import CASES
from test_attention_malformed import NARROW, check_light_weights, light_weights, narrow_problem
from test_gpu_attention import _attend

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


def test_serving_without_enough_blocks_raises():
    """The prefill of the first batch lacks blocks; the tokens behind it need none."""
    from test_gpu_attention_example import _example
    with pytest.raises(RuntimeError, match="missing"):
        _example().run(sessions=4, batch=4, dtype="f32", n_layers=1, d_model=64, n_q_heads=1, n_kv_heads=1, n_blocks=3, block_size=64,
                       prompt_len=(100, 101), user_len=(1, 2), out_len=(1, 2), capacity_bytes=1 << 20)


@pytest.mark.parametrize("scale", [8.3e-39, 1.3e-38, 2.4e-38])
@pytest.mark.parametrize("name", ["decode", "few_tokens_wide", "chunk", "f32"])
def test_attend_smallest_scales(name, scale):
    print(f"attend scale {name} {scale}", flush=True)
    p = ah.make(11, *CASES[name])
    p.scale = float(np.float32(scale))
    ah.check(p, *_attend(p), f"{name} {scale}")


@pytest.mark.parametrize("name", ["decode", "few_tokens_wide", "chunk_group", "f32"])
def test_attend_scores_beyond_fp32(name):
    """Rows whose scaled scores fp32 has no place for are NaN; none looks like a row that sees nothing."""
    print(f"attend beyond fp32 {name}", flush=True)
    p = ah.make(11, *CASES[name])
    p.scale = 1e38
    out, lse = _attend(p)
    assert not np.any(np.isneginf(lse)) and np.isnan(out).all(-1).mean() > 0.5


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("max_new,new", [(1, 1), (0, 40)])
def test_attend_many_light_keys(max_new, new, dtype):
    print(f"attend light keys {dtype} {new}", flush=True)
    p = light_weights(max_new, dtype, new=new)
    check_light_weights(p, *_attend(p), f"{dtype} {new}")


def test_what_is_written_gets_a_new_version():
    """Autograd keeps a cache (or `out`, q_out, a table) for a backward pass: written since, it is refused there as any tensor
    that was changed in place; what the calls only read stays as it is."""
    from paper_2411_19379_amd import attention as attn
    h = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device=DEV)
    table, free, n_free, cu, lens = z(1, 4), torch.arange(5, dtype=torch.int32, device=DEV), z(1) + 5, torch.tensor([0, 3], dtype=torch.int32, device=DEV), z(1)
    k_cache, v_cache, q, k = h(5, 2, 16, 64), h(5, 2, 16, 64), h(3, 4, 64), h(3, 2, 64)
    q_out, out = h(3, 4, 64), h(3, 4, 64)
    read = [free, n_free, cu, lens, q, k]
    w = torch.ones((), dtype=torch.bfloat16, device=DEV, requires_grad=True)
    losses = [(x * w).sum() for x in (k_cache, v_cache, q_out, out)]
    before, read_before = [x._version for x in (table, k_cache, v_cache, q_out, out)], [x._version for x in read]
    step = attn.assign_blocks(16, 3, cu, lens, table, free, n_free, in_place=True)
    attn.rope_append(q, k, k, step.positions, step.slots, None, k_cache, v_cache, q_out=q_out)
    attn.attend(q_out, k_cache, v_cache, step.table, cu, lens, out=out)
    assert all(x._version > b for x, b in zip((table, k_cache, v_cache, q_out, out), before))
    assert [x._version for x in read] == read_before
    for loss in losses:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    with torch.inference_mode():  # tensors without versions
        caches = h(5, 2, 16, 64), h(5, 2, 16, 64)
        made = h(3, 4, 64)
        attn.rope_append(q, k, k, step.positions, step.slots, None, *caches, q_out=made)
    attn.attend(made, *caches, step.table, cu, lens, out=made)
