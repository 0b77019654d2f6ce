"""Forward-mode differentiation: the operators hand on no tangents, so tensors that have one are refused instead of answered without."""
import os

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2411_19379_amd import attention as attn
from paper_2411_19379_amd import build as b
from paper_2411_19379_amd import recurrence as rec


@pytest.fixture(autouse=True, scope="module")
def bindings():
    if not os.path.exists(b.ATTN_BINDING_PATH):
        b.build_attention_binding()
    if not os.path.exists(b.REC_BINDING_PATH):
        b.build_recurrence_binding()


def _calls(device):
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=device)
    rows = lambda *s: torch.zeros(*s, device=device)
    heads, cache = rows(1, 2, 64), rows(2, 2, 16, 64)
    layer = dict(q=heads, k_cache=cache, v_cache=cache.clone(), table=ints(0).view(1, 1), cu_seqlens=ints(0, 1), cached_lens=ints(0))
    yield attn.rope_append, dict(q=heads, k=heads, v=heads, positions=ints(0), slots=ints(0).long(), rotary=rows(4, 2, 32), k_cache=cache, v_cache=cache.clone(),
                                 q_out=rows(1, 2, 64))
    yield attn.attend, dict(layer, out=rows(1, 2, 64))
    yield attn.attend_tree, dict(layer, positions=ints(0), seen=ints(1).view(1, 1), out=rows(1, 2, 64))
    yield (lambda cache, **kw: attn.keep_path([cache], **kw)), dict(cache=cache, table=layer["table"], cu_seqlens=ints(0, 1), cached_lens=ints(0), path=ints(0))
    x, one = [rows(1, 8) for _ in range(3)], ints(0, 1)
    gates = dict(x=x[0], r=x[1], i=x[2], decay=rows(8))
    yield rec.gated_scan, dict(gates, cu_seqlens=one, init_states=rows(1, 8), out=rows(1, 8))
    yield rec.gated_scan_grads, dict(gates, dy=rows(1, 8), d_final=rows(1, 8), cu_seqlens=one, init_states=rows(1, 8))
    yield rec.gated_step, dict(gates, states=rows(1, 8), out=rows(1, 8))
    yield rec.gated_step_tree, dict(gates, states=rows(1, 8), cu_seqlens=one, parents=ints(-1), out=rows(1, 8))
    yield rec.keep_states, dict(states=rows(1, 8), node_states=rows(1, 8), cu_seqlens=one, path=ints(0), counts=ints(1))


NAMES = ["rope_append", "attend", "attend_tree", "keep_path", "gated_scan", "gated_scan_grads", "gated_step", "gated_step_tree", "keep_states"]


def _check(which, device):
    call, args = list(_calls(device))[which]
    for name, t in args.items():
        if not t.dtype.is_floating_point:
            continue
        with forward_ad.dual_level():
            kw = dict(args, **{name: forward_ad.make_dual(t, torch.ones_like(t))})
            for mode in (torch.enable_grad, torch.no_grad):  # which does not stop forward mode
                with mode(), pytest.raises(ValueError, match="tangent"):
                    call(**kw)
            yield lambda: call(**dict(kw, **{name: kw[name].detach()}))


@pytest.mark.parametrize("which", range(len(NAMES)), ids=NAMES)
def test_tangents_are_not_dropped_in_silence(which):
    for detached in _check(which, "cpu"):
        with pytest.raises(ValueError, match="CUDA"):  # the next check: no host tensors
            detached()


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(len(NAMES)), ids=NAMES)
def test_tangents_on_the_gpu(which):
    for detached in _check(which, "cuda:0"):
        detached()


@pytest.mark.gpu
def test_a_graph_of_gradients_has_no_tangents():
    x, decay, cu = torch.zeros(1, 8, device="cuda:0"), torch.zeros(8, device="cuda:0", requires_grad=True), torch.tensor([0, 1], dtype=torch.int32, device="cuda:0")
    with forward_ad.dual_level(), pytest.raises((ValueError, NotImplementedError)):
        rec.gated_scan(forward_ad.make_dual(x, x), x, x, decay, cu)
