"""Problems for the gated recurrence and the bounds its results are held to, shared by the emulation and the GPU tests."""
from __future__ import annotations

from types import SimpleNamespace

import numpy as np
import torch

import rec_oracle

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CODE = {"f32": 0, "bf16": 1, "f16": 2}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def make(seed, C, dtype, lens, init=True, sharpness=8.0, lead=0, behind=0, spread=1.0, keep=(0.5, 0.999)):
    """Random inputs.  `lead` and `behind`: tokens of no sequence in front and behind, which hold NaN."""
    g = torch.Generator().manual_seed(seed)
    p = SimpleNamespace(C=C, dtype=dtype, lens=list(lens), sharpness=sharpness)
    p.cu = (np.concatenate([[0], np.cumsum(lens)]) + lead).astype(np.int32)
    p.T = int(p.cu[-1]) + behind
    rand = lambda *s: torch.randn(s, generator=g) * spread
    p.x, p.r, p.i, p.dy = (rand(p.T, C).to(TORCH[dtype]) for _ in range(4))
    for v in (p.x, p.r, p.i, p.dy):
        v[:lead] = float("nan")
        v[p.T - behind:] = float("nan")
    a = keep[0] + (keep[1] - keep[0]) * torch.rand(C, generator=g, dtype=torch.float64)
    p.decay = torch.log(torch.expm1(-a.log() / sharpness)).float()
    p.init = torch.randn((len(lens), C), generator=g) if init else None
    p.d_final = torch.randn((len(lens), C), generator=g)
    return p


def arrays(p):
    return [v.double().numpy() for v in (p.x, p.r, p.i)] + [p.decay.double().numpy()]


def reference(p):
    return rec_oracle.scan(*arrays(p), p.cu, p.sharpness, None if p.init is None else p.init.numpy())


# Error bounds, in units of half an ulp of 1 in fp32.  A product or a sum is off by 1 unit of itself, the hardware's exp2, reciprocal
# and (reciprocal) root by 2 (one ulp), expf and log1pf by 4.  To first order, and rounded up:
#
#   sigmoid(v) = 1 / (1 + 2^(-log2(e) v)): the exponent is off by 2 units of itself, the power by that times |v| and by 2, of which
#       1 - sigmoid reaches the sum; sum and reciprocal 3 more
#   rate = -sharpness softplus(decay) log2(e): 4 + 4 + 4;   log a = rate sigmoid: those of both and 1;   a: |log a| times that, and 2
#   1 - a^2: as log a and 5 more from the series, behind -2 log a = 1/4 twice a^2's share of a's and 1 of 1; its root half of that and 3
#   what is added, sqrt(1 - a^2) sigmoid(i) x: those of its factors and 2
#   a state: a times the error in front, the error of a and 4 more (a sum and a product as the tokens follow one another, and as many
#       for partial sums, each of which passes over tokens that are counted already) times the size in front, and what is added
#
# where "size" is the sum with all terms' sizes, so that every bound is the arithmetic's and none is fitted to a result.
UNIT = 2.0 ** -24


def _sigmoid_error(v):
    return (2 * np.abs(v) + 2) * (1 - rec_oracle.sigmoid(v)) + 3


class Errors:
    """Sizes and errors of every token's factors, relative to the factors."""

    def __init__(self, p):
        self.x, self.r, self.i, self.decay = arrays(p)
        x, r, i, decay = self.x, self.r, self.i, self.decay
        self.a, self.beta, self.sr, self.si, self.log_a = rec_oracle.parts(x, r, i, decay, p.sharpness)
        self.sr_off, self.si_off = _sigmoid_error(r), _sigmoid_error(i)
        self.log_off = 12 + self.sr_off + 1
        self.a_off = np.abs(self.log_a) * self.log_off + 2
        with np.errstate(divide="ignore", invalid="ignore"):
            square = np.where(-2 * self.log_a < 0.26, self.log_off + 5, (2 * self.a ** 2 * self.a_off + 2) / self.beta ** 2)
        self.beta_off = square / 2 + 3
        self.added = self.beta * self.si * np.abs(x)
        self.added_off = self.beta_off + self.si_off + 2

    def states(self, p):
        """Sizes and errors of the states of all tokens and of those in front of them."""
        size, off, size_before, off_before = (np.zeros(self.a.shape) for _ in range(4))
        for b in range(len(p.lens)):
            s = np.zeros(p.C) if p.init is None else np.abs(p.init[b].double().numpy())
            e = np.zeros(p.C)
            for t in range(p.cu[b], p.cu[b + 1]):
                size_before[t], off_before[t] = s, e
                e = self.a[t] * (e + (self.a_off[t] + 4) * s) + self.added_off[t] * self.added[t]
                s = self.a[t] * s + self.added[t]
                size[t], off[t] = s, e
        return size, off, size_before, off_before

    def behind(self, p, dy, d_final):
        """The same for the gradients of the states, and of the initial ones."""
        size, off = np.zeros(self.a.shape), np.zeros(self.a.shape)
        size_init, off_init = np.zeros((len(p.lens), p.C)), np.zeros((len(p.lens), p.C))
        for b in range(len(p.lens)):
            s = np.zeros(p.C) if d_final is None else np.abs(d_final[b])
            e = np.zeros(p.C)
            for t in range(p.cu[b + 1] - 1, p.cu[b] - 1, -1):
                s = s + (0.0 if dy is None else np.abs(dy[t]))
                e = e + s
                size[t], off[t] = s, e
                e = self.a[t] * (e + (self.a_off[t] + 4) * s)
                s = self.a[t] * s
            size_init[b], off_init[b] = s, e
        return size, off, size_init, off_init


def check(what, got, want, bound):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), f"{what}: not finite in other places than the definition"
    fine = np.isfinite(want)
    far = np.where(fine, np.abs(np.where(fine, got, 0) - np.where(fine, want, 0)) / np.where(fine, np.broadcast_to(bound, want.shape), 1), 0.0)
    worst = float(far.max()) if far.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times the bound at {np.unravel_index(far.argmax(), far.shape)}"
    return worst


def check_scan(p, y, final, ckpt=None, ckpt_states=None):
    h, want_final = reference(p)
    _, off, _, _ = Errors(p).states(p)
    bound = off * UNIT + 1e-30
    inside = slice(int(p.cu[0]), int(p.cu[-1]))
    tiny = 2.0 ** -25 if p.dtype == "f16" else 1e-38  # half the smallest step of fp16
    check("y", y[inside], h[inside], (bound + HALF_ULP[p.dtype] * (np.abs(h) + bound) + tiny)[inside])
    init = np.zeros((len(p.lens), p.C)) if p.init is None else p.init.double().numpy()
    for b, n in enumerate(p.lens):
        if n:
            check("final", np.asarray(final)[b], want_final[b], bound[p.cu[b + 1] - 1])
        else:
            assert np.array_equal(np.asarray(final)[b], init[b].astype(np.float32))
    if ckpt is not None:
        ok = (np.asarray(ckpt) >= p.cu[0]) & (np.asarray(ckpt) < p.cu[-1])
        at = np.where(ok, ckpt, 0)
        check("ckpt", ckpt_states, np.where(ok[:, None], h[at], 0.0), np.where(ok[:, None], bound[at], 1e-30))


def check_grads(p, got, dy=True, d_final=True, init=True):
    dy_of, d_final_of = p.dy.double().numpy() if dy else None, p.d_final.double().numpy() if d_final else None
    want = rec_oracle.grads(*arrays(p), p.cu, p.sharpness, None if p.init is None else p.init.double().numpy(), dy_of, d_final_of)
    e = Errors(p)
    _, _, before, before_off = e.states(p)
    G, G_off, size_init, init_off = e.behind(p, dy_of, d_final_of)
    inside = np.zeros((p.T, 1), bool)
    inside[p.cu[0]:p.cu[-1]] = True
    half, tiny = HALF_ULP[p.dtype], 2.0 ** -25 if p.dtype == "f16" else 1e-38
    with np.errstate(divide="ignore", invalid="ignore"):
        over = np.where(e.beta > 0, 1.0 / e.beta, 0.0)
        # 1 - sigmoid: sigmoid's error, and 1 unit
        si_rest, sr_rest = (off * s / (1 - s) + 1 for off, s in ((e.si_off, e.si), (e.sr_off, e.sr)))
        second = e.a ** 2 * over * e.si * np.abs(e.x)
        inner = e.a * before + second
        inner_off = e.a * (before_off + (e.a_off + 1) * before) + (2 * e.a_off + e.beta_off + e.si_off + 5) * second + inner
        d_log, d_log_off = G * inner, G_off * inner + G * inner_off + G * inner
        add = e.beta * e.si
        dx = (G * add, G_off * add + (e.beta_off + e.si_off + 4) * G * add)
        x = np.abs(e.x) * (1 - e.si)
        di = (dx[0] * x, dx[1] * x + (si_rest + 4) * dx[0] * x)
        w = np.abs(e.log_a) * (1 - e.sr)
        dr = (d_log * w, d_log_off * w + (e.log_off + 2 + sr_rest + 2) * d_log * w)
    for what, g, exact, (size, off) in (("dx", got[0], want[0], dx), ("dr", got[1], want[1], dr), ("di", got[2], want[2], di)):
        off, exact = np.where(inside, off * UNIT, 0.0), np.where(inside, exact, 0.0)
        check(what, g, exact, off + half * (np.abs(exact) + off) + tiny)
    # a chunk's sum in 15 roundings, then 64 bits; its factor 8 units
    per_token = np.where(inside, d_log_off * e.sr + (e.sr_off + 1 + 15 + 8) * d_log * e.sr, 0.0)
    check("d_decay", got[3], want[3], UNIT * per_token.sum(0) * p.sharpness * rec_oracle.sigmoid(e.decay) + 1e-30)
    if init:
        check("d_init", got[4], want[4], UNIT * init_off + 1e-30)


# channels, type, lengths, and more
CASES = {
    "one_token": (64, "bf16", [1], {}),
    "one_channel": (1, "f32", [5, 0, 70], {}),
    "odd": (67, "bf16", [3, 130, 0, 1], dict(init=False)),
    "chunks": (128, "f16", [64, 128, 63, 1, 65], {}),
    "many_short": (40, "f32", [1, 2, 0, 3, 1, 1, 7, 0, 0, 16, 17, 1], {}),
    "groups": (66, "bf16", [1100, 40], {}),
    "groups_f32": (130, "f32", [2000], dict(init=False)),
    "lead_and_behind": (32, "f32", [50, 100], dict(lead=7, behind=80)),
    "none_at_all": (32, "bf16", [0, 0], dict(behind=70)),
}
