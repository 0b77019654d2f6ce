"""The attention operators have no backward pass: tensors that require grad are refused where a graph would be recorded."""
import os

import pytest
import torch

from paper_2411_19379_amd import attention as attn
from paper_2411_19379_amd import build as b


@pytest.fixture(autouse=True, scope="module")
def binding():
    if not os.path.exists(b.ATTN_BINDING_PATH):
        b.build_attention_binding()


def _calls():
    ints = torch.zeros(2, dtype=torch.int32)
    x, cache = torch.zeros(1, 2, 64), torch.zeros(2, 2, 16, 64)
    table = torch.zeros(4, 2, 32)
    yield attn.rope_append, dict(q=x, k=x, v=x, positions=ints[:1], slots=ints[:1].long(), rotary=table, k_cache=cache, v_cache=cache, q_out=x)
    yield attn.attend, dict(q=x, k_cache=cache, v_cache=cache, table=ints.view(1, 2), cu_seqlens=ints, cached_lens=ints[:1], out=x)


@pytest.mark.parametrize("call,args", [pytest.param(f, a, id=f.__name__) for f, a in _calls()])
def test_gradients_are_not_dropped_in_silence(call, args):
    for name, t in args.items():
        if not t.dtype.is_floating_point:
            continue
        kw = dict(args, **{name: t.clone().requires_grad_()})
        with pytest.raises(ValueError, match=f"{name} requires grad"):
            call(**kw)
        for mode in (torch.no_grad, torch.inference_mode):
            with mode(), pytest.raises(ValueError, match="CUDA"):  # the next check: no host tensors
                call(**kw)
