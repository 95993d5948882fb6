"""How far a result of the sequence operators may be from the oracle's, element by element, from the number formats alone.

u is the unit roundoff of the result's type (half the distance of neighbouring values), E that of fp32.  An fp32 sum of magnitudes that add
up to s, in whatever order, with at most k additions in a row behind each term is within k E s.  K covers the additions and the few
operations around them: 64 where sums are trees over a row, more where a number of terms comes in."""
from __future__ import annotations

import numpy as np

from oracle import sequence as S

E = 2.0 ** -24
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}         # 2^-p of a significand of p bits: 24, 11, 8
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}   # below it a result may become zero or lose places
K = 64


def rounded(exp, before, dtype):
    """`exp` computed to within `before`, then rounded once."""
    return before + U[dtype] * (np.abs(exp) + before) + TINY[dtype]


def _norm(x, eps):
    d = x - x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    err = K * E * ((np.abs(x) + np.abs(x).mean(1, keepdims=True)) * rstd + np.abs(d) * rstd)   # of xh
    # an error of the mean shifts the whole row: it reaches the variance through the deviations
    err = err + np.abs(d) * rstd * (err * np.abs(d) * rstd).mean(1, keepdims=True)
    return d * rstd, rstd, err


def layernorm(x, gamma, beta, eps, dtype):
    xh, _, err = _norm(x, eps)
    return rounded(xh * gamma + beta, err * np.abs(gamma) + 4 * E * (np.abs(xh * gamma) + np.abs(beta)), dtype)


def layernorm_backward(x, gamma, eps, dy, add, dtype):
    xh, rstd, err = _norm(x, eps)
    q, m = np.abs(dy * gamma), lambda v: v.mean(1, keepdims=True)
    inner = K * E * (q + m(q) + np.abs(xh) * m(q * np.abs(xh))) + err * m(q * np.abs(xh)) + np.abs(xh) * m(q * err)
    size = rstd * (q + m(q) + np.abs(xh) * m(q * np.abs(xh)))
    spread = (err * np.abs(xh)).mean(1, keepdims=True)                     # relative error of rstd
    dx, dg, db = S.layernorm_backward(x, gamma, eps, dy)
    rows = 64 + len(x) ** 0.5
    return (rounded(dx + add, rstd * inner + size * (spread + K * E) + 2 * E * np.abs(add), dtype),
            (np.abs(dy) * (err + rows * E * np.abs(xh))).sum(0) + TINY["f32"], (np.abs(dy) * rows * E).sum(0) + TINY["f32"])


def _scan(off, backwards, n_seq, start, step):
    for s in range(n_seq):
        rows = S._rows(off, s, backwards)
        v = start[s]
        for i, t in enumerate(rows):
            v = step(s, rows, i, t, v)


def recurrence(x, gate, off, h0, backwards, dtype):
    """Bounds of (y, last): each step adds K E (1 + |gate|) of its terms' size -- the gate's exponent is exact to E |gate| --, and the state's error
    travels on through the gate."""
    a, take = S.sigmoid(gate), S.sigmoid(-gate)
    y, _ = S.recurrence(x, gate, off, h0, backwards)
    err, last = np.zeros_like(x), np.zeros_like(h0)

    def step(s, rows, i, t, v):
        before = np.abs(y[rows[i - 1]] if i else h0[s])
        err[t] = a[t] * v + K * E * (1 + np.abs(gate[t])) * (a[t] * before + take[t] * np.abs(x[t]))
        last[s] = err[t]
        return err[t]

    _scan(off, backwards, len(off) - 1, np.zeros_like(h0), step)
    return rounded(y, err, dtype), last + TINY["f32"], err


def recurrence_backward(x, gate, off, h0, dy, dlast, backwards, dtype):
    a, take = S.sigmoid(gate), S.sigmoid(-gate)
    y, _ = S.recurrence(x, gate, off, h0, backwards)
    dx, dg, _ = S.recurrence_backward(x, gate, off, h0, dy, dlast, backwards)
    _, _, eh = recurrence(x, gate, off, h0, backwards, dtype)
    bx, bg, b0 = np.zeros_like(x), np.zeros_like(x), np.zeros_like(h0)
    for s in range(len(off) - 1):
        rows = S._rows(off, s, backwards)
        v, u_next = np.zeros(x.shape[1]), np.abs(dlast[s])
        flow = dlast[s]
        for i in reversed(range(len(rows))):
            t = rows[i]
            u = dy[t] + flow
            eu = v + K * E * (np.abs(dy[t]) + u_next)
            rel = K * E * (1 + np.abs(gate[t]))
            before = y[rows[i - 1]] if i else h0[s]
            e_before = eh[rows[i - 1]] if i else 0.0
            bx[t] = take[t] * (eu + rel * np.abs(u))
            at = a[t] * take[t]
            bg[t] = at * (np.abs(before - x[t]) * (eu + rel * np.abs(u)) + np.abs(u) * (e_before + 2 * E * (np.abs(before) + np.abs(x[t]))))
            flow = a[t] * u
            v = a[t] * eu + rel * np.abs(flow)
            u_next = np.abs(flow)
        b0[s] = v
    return rounded(dx, bx, dtype), rounded(dg, bg, dtype), b0 + TINY["f32"]


def _products(act, x, wg, wu):
    """(G, U, H, their bounds) of the two products and the activation, whose slope stays below 1.2."""
    k = (16 + x.shape[1]) * E
    g, up = x @ wg, x @ wu
    eg, eu = k * (np.abs(x) @ np.abs(wg)), k * (np.abs(x) @ np.abs(wu))
    value, slope = S.activate(act, g)
    ev = 1.2 * eg + 16 * E * (1 + np.abs(g)) * np.abs(value) + TINY["f32"]
    return g, up, value, slope, eg, eu, ev


def ffn(act, x, wg, wu, wd, res, dtype):
    _, up, value, _, _, eu, ev = _products(act, x, wg, wu)
    h = value * up
    eh = ev * np.abs(up) + np.abs(value) * eu + U[dtype] * np.abs(h) + TINY[dtype]
    y = h @ wd + res
    return rounded(y, eh @ np.abs(wd) + (16 + wd.shape[0]) * E * (np.abs(h) @ np.abs(wd)) + 2 * E * np.abs(res), dtype)


def ffn_backward(act, x, wg, wu, wd, dy, dtype):
    g, up, value, slope, eg, eu, ev = _products(act, x, wg, wu)
    dh = dy @ wd.T
    edh = (16 + x.shape[1]) * E * (np.abs(dy) @ np.abs(wd.T))
    es = 1.2 * eg + 32 * E * (1 + np.abs(g) ** 2) * (np.abs(slope) + 0.01)          # the slope's own slope stays below 1.2
    h, dg, du = value * up, dh * up * slope, dh * value
    eh = ev * np.abs(up) + np.abs(value) * eu + U[dtype] * np.abs(h) + TINY[dtype]
    edg = edh * np.abs(up * slope) + np.abs(dh * slope) * eu + np.abs(dh * up) * es + (U[dtype] + 4 * E) * np.abs(dg) + TINY[dtype]
    edu = edh * np.abs(value) + np.abs(dh) * ev + (U[dtype] + 4 * E) * np.abs(du) + TINY[dtype]
    kf, kn, xa, dya = (16 + 2 * wd.shape[0]) * E, (16 + len(x)) * E, np.abs(x), np.abs(dy)
    dx, dwg, dwu, dwd = S.ffn_backward(act, x, wg, wu, wd, dy)
    return (rounded(dx, (edg + kf * np.abs(dg)) @ np.abs(wg.T) + (edu + kf * np.abs(du)) @ np.abs(wu.T), dtype),
            rounded(dwg, xa.T @ (edg + kn * np.abs(dg)), dtype), rounded(dwu, xa.T @ (edu + kn * np.abs(du)), dtype),
            rounded(dwd, (eh + kn * np.abs(h)).T @ dya, dtype))
