"""Plain float64 definitions of the sequence operators (numpy, row by row where the definition is): layer norm, gated linear
recurrence, gated feed-forward network, and their gradients written out from the chain rule."""
from __future__ import annotations

import math

import numpy as np


def sigmoid(z):
    """1 / (1 + exp(-z)) without overflow."""
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1 / (1 + e), e / (1 + e))


def frame_offsets(coords, n_batch):
    """First row of every frame of a voxel list sorted by frame, and the number of rows."""
    return np.array([int((coords[:, 0] < b).sum()) if b else 0 for b in range(n_batch)] + [len(coords)])


def layernorm(x, gamma, beta, eps):
    d = x - x.mean(1, keepdims=True)
    return d / np.sqrt((d * d).mean(1, keepdims=True) + eps) * gamma + beta


def layernorm_backward(x, gamma, eps, dy):
    """(dx, dgamma, dbeta)"""
    d = x - x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    xh, q = d * rstd, dy * gamma
    dx = rstd * (q - q.mean(1, keepdims=True) - xh * (q * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def _rows(offsets, s, backwards):
    rows = range(int(offsets[s]), int(offsets[s + 1]))
    return list(reversed(rows)) if backwards else list(rows)


def recurrence(x, gate, offsets, h0, backwards=False):
    """(y, last states); h0 [sequences][channels]."""
    a, take = sigmoid(gate), sigmoid(-gate)
    y, last = np.zeros_like(x), h0.copy()
    for s in range(len(offsets) - 1):
        for t in _rows(offsets, s, backwards):
            last[s] = a[t] * last[s] + take[t] * x[t]
            y[t] = last[s]
    return y, last


def recurrence_backward(x, gate, offsets, h0, dy, dlast, backwards=False):
    """(dx, dgate, dh0)"""
    a, take = sigmoid(gate), sigmoid(-gate)
    y, _ = recurrence(x, gate, offsets, h0, backwards)
    dx, dgate, dh0 = np.zeros_like(x), np.zeros_like(x), dlast.copy()
    for s in range(len(offsets) - 1):
        rows = _rows(offsets, s, backwards)
        for i in reversed(range(len(rows))):
            t = rows[i]
            u = dy[t] + dh0[s]
            before = y[rows[i - 1]] if i else h0[s]
            dx[t] = take[t] * u
            dgate[t] = u * (before - x[t]) * a[t] * take[t]
            dh0[s] = a[t] * u
    return dx, dgate, dh0


def activate(act, g):
    """(act(g), its derivative); act "silu" or "gelu" (the tanh form)."""
    if act == "silu":
        s = sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    k = math.sqrt(2 / math.pi)
    t = np.tanh(k * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def ffn(act, x, wg, wu, wd):
    return (activate(act, x @ wg)[0] * (x @ wu)) @ wd


def ffn_backward(act, x, wg, wu, wd, dy):
    """(dx, dwg, dwu, dwd)"""
    value, slope = activate(act, x @ wg)
    up, dh = x @ wu, dy @ wd.T
    dg, du = dh * up * slope, dh * value
    return dg @ wg.T + du @ wu.T, x.T @ dg, x.T @ du, (value * up).T @ dy
