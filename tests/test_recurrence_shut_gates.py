"""The gated recurrence where gates are nearly shut and decays nearly nothing, so that 1 - a^2 lies around the smallest normal number:
scan, single tokens and gradients against the definition in 64 bits, on the emulator with the instructions' treatment of denormals and
on the GPU."""
from __future__ import annotations

import os

import numpy as np
import pytest
import torch

import rec_helpers as rh
import rec_oracle
import test_recurrence_emulation as emulation
from paper_2411_19379_amd import recurrence as rec

DEV = "cuda:0"
SMALLEST = 2.0 ** -126  # the smallest normal number


@pytest.fixture(scope="session")
def emu(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("rec_emu_denormals"))
    os.mkdir(os.path.join(d, "hip"))  # found in front of rec_emu's
    with open(os.path.join(d, "hip", "hip_runtime.h"), "w") as f:
        f.write(f'#include "{os.path.join(emulation.HERE, "denormals.h")}"\n')
    return emulation._build(d, 0)


# Beside the roundings that rec_helpers counts:  exp2, reciprocal and roots take operands and results below SMALLEST as 0, so sigmoid,
# softplus, log a, 1 - a^2 and products of them may be lost where they are that small.  With s the sharpness, 1 - a^2 <= 2 s softplus(decay)
# sigmoid(r), so where one of them is lost sqrt(1 - a^2) is at most LOST = sqrt(2 s max(1, softplus(decay)) SMALLEST), and that is the
# most by which it is off.  What is off by that, or less:
#
#   what is added to the state    LOST sigmoid(i) |x|, or SMALLEST |x| where sigmoid(i) is lost;   states: the sum of it, times a
#   dx, di                        the gradient of the state times LOST sigmoid(i), and |x| (1 - sigmoid(i))
#   dr, d_decay                   their part through sqrt(1 - a^2) is that gradient times a^2 sigmoid(i) |x| |log a| / sqrt(1 - a^2), and
#                                 |log a| / sqrt(1 - a^2) <= LOST there;   their other part the gradient times what the state in front is
#                                 off by, and with |log a| lost the gradient and the state times s max(1, softplus(decay)) SMALLEST
def check(p, y, final, got=None, dy=True):
    e = rh.Errors(p)
    grew = np.maximum(1.0, np.logaddexp(0.0, e.decay))
    LOST = np.sqrt(2 * p.sharpness * grew * SMALLEST)
    x = np.abs(e.x)
    size, off, before, before_off = e.states(p)
    lost, lost_before = np.zeros(e.a.shape), np.zeros(e.a.shape)
    for b in range(len(p.lens)):
        behind = np.zeros(p.C)
        for t in range(p.cu[b], p.cu[b + 1]):
            lost_before[t] = behind
            behind = e.a[t] * behind + (LOST * e.si[t] + SMALLEST) * x[t] + p.sharpness * grew * SMALLEST * before[t]
            lost[t] = behind
    bound = off * rh.UNIT + lost + 1e-30
    half, tiny = rh.HALF_ULP[p.dtype], 2.0 ** -25 if p.dtype == "f16" else 1e-38
    h, want_final = rh.reference(p)
    rh.check("y", y, h, bound + half * (np.abs(h) + bound) + tiny)
    for b, n in enumerate(p.lens):
        if n:
            rh.check("final", np.asarray(final)[b], want_final[b], bound[p.cu[b + 1] - 1])
    if got is None:
        return
    dy_of, d_final = p.dy.double().numpy() if dy else None, p.d_final.double().numpy()
    want = rec_oracle.grads(*rh.arrays(p), p.cu, p.sharpness, p.init.double().numpy(), dy_of, d_final)
    G, G_off, _, init_off = e.behind(p, dy_of, d_final)
    with np.errstate(divide="ignore", invalid="ignore"):
        second = np.where(e.beta > 0, e.a ** 2 / e.beta, 0.0) * e.si * x
    log_a = np.abs(e.log_a)
    inner = e.a * before + second
    inner_off = e.a * (before_off + (e.a_off + 1) * before) + (2 * e.a_off + e.beta_off + e.si_off + 5) * second + inner
    d_log, d_log_off = G * inner, G_off * inner + G * inner_off + G * inner
    dropped = G * ((LOST * e.si + SMALLEST) * x + lost_before * log_a + p.sharpness * grew * SMALLEST * before)
    add = e.beta * e.si
    dx = G * add
    dx_off = G_off * add + (e.beta_off + e.si_off + 4) * dx
    # 1 - sigmoid is off by what sigmoid is, and by 1 unit of itself
    di_off = dx_off * x * (1 - e.si) + (e.si_off * e.si + 5 * (1 - e.si)) * dx * x
    dr_off = (d_log_off + (e.log_off + 4) * d_log) * log_a * (1 - e.sr) + (e.sr_off * e.sr + 1 - e.sr) * d_log * log_a
    lost_dx = G * (LOST * e.si + SMALLEST)
    for what, g, exact, by in (("dx", got[0], want[0], dx_off * rh.UNIT + lost_dx), ("dr", got[1], want[1], dr_off * rh.UNIT + dropped),
                               ("di", got[2], want[2], di_off * rh.UNIT + lost_dx * x)):
        rh.check(what, g, exact, by + half * (np.abs(exact) + by) + tiny)
    per_token = (d_log_off + (e.sr_off + 1 + 15 + 8) * d_log) * e.sr
    rh.check("d_decay", got[3], want[3], rh.UNIT * per_token.sum(0) * p.sharpness * rec_oracle.sigmoid(e.decay) + dropped.sum(0) + 1e-30)
    rh.check("d_init", got[4], want[4], rh.UNIT * init_off + 1e-30)


def _shut(dtype, C, lens):
    """r from -120 to 30, i from -100 to 100, states that are kept at 0.9 to 0.9999 per token with an open gate."""
    p = rh.make(9, C, dtype, lens, keep=(0.9, 0.9999))
    n = torch.arange(p.T)
    p.r[:] = torch.where(n % 2 == 0, torch.linspace(-120.0, 30.0, p.T), torch.linspace(-92.0, -76.0, p.T))[:, None] + torch.linspace(0.0, 0.25, C)
    p.i[:] = torch.linspace(-100.0, 100.0, C)[torch.randperm(C, generator=torch.Generator().manual_seed(1))]
    p.i[n % 4 < 2] = 0.5
    p.dy[n % 3 == 0] = 0.0
    return p


def _slow(dtype, C, lens):
    """Ordinary gates, decays down to -90."""
    p = rh.make(10, C, dtype, lens)
    p.decay[:] = torch.linspace(-90.0, 4.0, C)
    p.dy[torch.arange(p.T) % 3 == 0] = 0.0
    return p


def _no_gradient(dtype, C, lens):
    """Nearly shut gates behind which no gradient comes: its product with what is infinite would be NaN."""
    p = _shut(dtype, C, lens)
    p.dy.zero_(), p.d_final.zero_()
    return p


PROBLEMS = [_shut, _slow, _no_gradient]
on_problems = pytest.mark.parametrize("problem", PROBLEMS, ids=lambda f: f.__name__[1:])


@on_problems
@pytest.mark.parametrize("dtype,C,lens", [("f32", 64, [60]), ("bf16", 66, [40, 0, 100]), ("f16", 130, [70])])
def test_emulated(emu, tmp_path, problem, dtype, C, lens):
    p = problem(dtype, C, lens)
    y, final, _, _ = emulation._scan(emu, tmp_path, p)
    check(p, y, final, emulation._grads(emu, tmp_path, p))


@pytest.mark.gpu
@on_problems
@pytest.mark.parametrize("dtype,C,lens", [("f32", 64, [60]), ("bf16", 66, [40, 0, 100]), ("f16", 130, [700, 31]), ("bf16", 2560, [500, 40]), ("f16", 2560, [530]),
                                          ("f32", 2560, [300])])
def test_on_the_gpu(problem, dtype, C, lens):
    p = problem(dtype, C, lens)
    x, r, i, decay, init, dy, d_final = (t.to(DEV) for t in (p.x, p.r, p.i, p.decay, p.init, p.dy, p.d_final))
    cu = torch.as_tensor(p.cu, device=DEV)
    numpy = lambda ts: [t.detach().double().cpu().numpy() for t in ts]
    out = rec.gated_scan(x, r, i, decay, cu, init_states=init)
    again = rec.gated_scan_grads(dy, d_final, x, r, i, decay, cu, init_states=init)
    check(p, *numpy(out[:2]), numpy(again))
    leaves = [t.clone().requires_grad_() for t in (x, r, i, decay, init)]
    out = rec.gated_scan(*leaves[:4], cu, init_states=leaves[4])
    for a, b in zip(torch.autograd.grad((out.y, out.final), leaves, (dy, d_final)), again):
        assert torch.equal(a, b)


@pytest.mark.gpu
@on_problems
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_tokens_on_the_gpu(problem, dtype):
    """A token of every sequence, and trees that are one token each."""
    p = problem(dtype, 130, [1] * 64)
    x, r, i, decay, states = (t.to(DEV) for t in (p.x, p.r, p.i, p.decay, p.init))
    cu = torch.as_tensor(p.cu, device=DEV)
    numpy = lambda t: t.double().cpu().numpy()
    y, nodes = rec.gated_step_tree(x, r, i, decay, states, cu, torch.full((64,), -1, dtype=torch.int32, device=DEV))
    check(p, numpy(y), numpy(nodes))
    y = rec.gated_step(x, r, i, decay, states)
    check(p, numpy(y), numpy(states))
