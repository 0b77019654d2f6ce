"""The gated recurrence from its definition in 64 bits, token by token, and its gradients from the chain rule written out token by
token.  Nothing here knows chunks."""
from __future__ import annotations

import numpy as np


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-np.asarray(v, np.float64)))


def parts(x, r, i, decay, sharpness):
    """a, beta = sqrt(1 - a^2), the sigmoids and log a of every token."""
    x, r, i, decay = (np.asarray(v, np.float64) for v in (x, r, i, decay))
    log_a = -sharpness * np.logaddexp(0.0, decay) * sigmoid(r)
    return np.exp(log_a), np.sqrt(-np.expm1(2.0 * log_a)), sigmoid(r), sigmoid(i), log_a


def scan(x, r, i, decay, cu, sharpness, init=None):
    """States of all tokens [T, C] (zeros for tokens of no sequence) and final states."""
    a, beta, _, si, _ = parts(x, r, i, decay, sharpness)
    b = beta * si * np.asarray(x, np.float64)
    batch, C = len(cu) - 1, len(decay)
    h, final = np.zeros(a.shape), np.zeros((batch, C))
    for s in range(batch):
        state = np.zeros(C) if init is None else np.asarray(init[s], np.float64)
        for t in range(cu[s], cu[s + 1]):
            state = a[t] * state + b[t]
            h[t] = state
        final[s] = state
    return h, final


def tree(x, r, i, decay, states, cu, parents, sharpness):
    a, beta, _, si, _ = parts(x, r, i, decay, sharpness)
    b = beta * si * np.asarray(x, np.float64)
    h = np.zeros(a.shape)
    for s in range(len(cu) - 1):
        for k in range(cu[s + 1] - cu[s]):
            p = parents[cu[s] + k]
            h[cu[s] + k] = a[cu[s] + k] * (h[cu[s] + p] if 0 <= p < k else np.asarray(states[s], np.float64)) + b[cu[s] + k]
    return h


def grads(x, r, i, decay, cu, sharpness, init, dy, d_final):
    """dx, dr, di, d_decay, d_init, and the sum of the sizes of what d_decay adds up."""
    a, beta, sr, si, log_a = parts(x, r, i, decay, sharpness)
    x, decay = np.asarray(x, np.float64), np.asarray(decay, np.float64)
    h, _ = scan(x, r, i, decay, cu, sharpness, init)
    batch, C = len(cu) - 1, len(decay)
    dx, dr, di = (np.zeros(a.shape) for _ in range(3))
    per_token = np.zeros(a.shape)
    d_init = np.zeros((batch, C))
    for s in range(batch):
        q = np.zeros(C) if d_final is None else np.asarray(d_final[s], np.float64).copy()
        for t in range(cu[s + 1] - 1, cu[s] - 1, -1):
            g = q + (0.0 if dy is None else np.asarray(dy[t], np.float64))
            before = h[t - 1] if t > cu[s] else np.zeros(C) if init is None else np.asarray(init[s], np.float64)
            dx[t] = g * beta[t] * si[t]
            di[t] = g * beta[t] * x[t] * si[t] * (1.0 - si[t])
            with np.errstate(divide="ignore", invalid="ignore"):
                d_log = g * (a[t] * before - np.where(beta[t] > 0, a[t] ** 2 / beta[t], 0.0) * si[t] * x[t])
            dr[t] = d_log * log_a[t] * (1.0 - sr[t])
            per_token[t] = d_log * sr[t]
            q = a[t] * g
        d_init[s] = q
    factor = -sharpness * sigmoid(decay)
    return dx, dr, di, per_token.sum(0) * factor, d_init, np.abs(per_token).sum(0) * np.abs(factor)
