"""Gated scans long enough for every level at which chunks hand on what is in front of them (chunks, groups of 8, 8 groups), on the GPU:
sequences that end and begin in the middle of each, checkpoints all over, gradients with and without saved states."""
import numpy as np
import pytest
import torch

import rec_helpers as rh
from paper_2411_19379_amd import recurrence as rec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# 8192 tokens are 8 groups forwards, 4096 backwards
@pytest.mark.parametrize("C,dtype,lens,keep", [(66, "bf16", [33000], (0.5, 0.999)), (64, "f32", [8192, 1, 8191, 0, 4096, 5000], (0.9, 0.9999)),
                                               (130, "f16", [9000, 100, 16, 12000], (0.5, 0.999)), (640, "bf16", [3, 17000], (0.99, 0.99999))])
def test_long(C, dtype, lens, keep):
    p = rh.make(23, C, dtype, lens, keep=keep)
    x, r, i, decay, init, dy, d_final = (t.to(DEV) for t in (p.x, p.r, p.i, p.decay, p.init, p.dy, p.d_final))
    cu = torch.as_tensor(p.cu, device=DEV)
    ckpt = np.random.RandomState(4).randint(-2, p.T + 2, 300).astype(np.int32)
    numpy = lambda ts: [t.detach().double().cpu().numpy() for t in ts]
    out = rec.gated_scan(x, r, i, decay, cu, init_states=init, ckpt=torch.as_tensor(ckpt, device=DEV))
    rh.check_scan(p, *numpy(out[:2]), ckpt, *numpy(out[2:]))
    got = rec.gated_scan_grads(dy, d_final, x, r, i, decay, cu, init_states=init)
    rh.check_grads(p, numpy(got))
    leaves = [t.clone().requires_grad_() for t in (x, r, i, decay, init)]
    again = rec.gated_scan(*leaves[:4], cu, init_states=leaves[4])
    assert torch.equal(again.y, out.y) and torch.equal(again.final, out.final)
    for a, b in zip(torch.autograd.grad((again.y, again.final), leaves, (dy, d_final)), got):
        assert torch.equal(a, b)
