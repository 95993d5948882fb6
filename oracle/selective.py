"""Plain float64 definitions of the selective state space operators (numpy, row by row where the definition is): short causal convolution, selective
scan, gated residual with its norms, and their gradients written out from the chain rule."""
from __future__ import annotations

import numpy as np

from .sequence import _rows, activate, sigmoid


def _history(x, before, rows, i, k, s):
    """x of k rows before the i-th of a sequence's rows."""
    return x[rows[i - k]] if i >= k else before[s, before.shape[1] + i - k]


def causal_conv(x, w, bias, offsets, before, silu=True, backwards=False):
    """(y, rows kept); w [taps][channels], before [sequences][taps - 1][channels], oldest first."""
    taps = len(w)
    y, last = np.zeros_like(x), before.copy()
    for s in range(len(offsets) - 1):
        rows = _rows(offsets, s, backwards)
        for i, t in enumerate(rows):
            z = bias + sum(w[k] * _history(x, before, rows, i, k, s) for k in range(taps))
            y[t] = activate("silu", z)[0] if silu else z
        everything = np.concatenate([before[s], x[rows]]) if rows else before[s]
        last[s] = everything[len(everything) - (taps - 1):]
    return y, last


def causal_conv_backward(x, w, bias, offsets, before, dy, dlast, silu=True, backwards=False):
    """(dx, dw, dbias, dbefore)"""
    taps = len(w)
    dx, dw, db, dbefore = np.zeros_like(x), np.zeros_like(w), np.zeros_like(bias), np.zeros_like(before)
    for s in range(len(offsets) - 1):
        rows = _rows(offsets, s, backwards)
        flow = np.zeros((taps - 1 + len(rows), x.shape[1]))              # of [before; x]
        for i, t in enumerate(rows):
            z = bias + sum(w[k] * _history(x, before, rows, i, k, s) for k in range(taps))
            dz = dy[t] * (activate("silu", z)[1] if silu else 1.0)
            db += dz
            for k in range(taps):
                dw[k] += dz * _history(x, before, rows, i, k, s)
                flow[taps - 1 + i - k] += w[k] * dz
        flow[len(rows):] += dlast[s]
        dbefore[s] = flow[:taps - 1]
        if rows:
            dx[rows] = flow[taps - 1:]
    return dx, dw, db, dbefore


def softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def selective_scan(x, dt, a, b, c, offsets, h0, skip, dt_bias, backwards=False, seen=None):
    """(y, last states); a [channels][states], h0 [sequences][channels][states].  seen(t, s, i, before, after): the states of every row."""
    d = softplus(dt + dt_bias)
    y, last = skip * x, h0.copy()
    for s in range(len(offsets) - 1):
        for i, t in enumerate(_rows(offsets, s, backwards)):
            before = last[s].copy()
            last[s] = np.exp(d[t][:, None] * a) * before + (d[t] * x[t])[:, None] * b[t]
            y[t] += last[s] @ c[t]
            if seen:
                seen(t, s, i, before, last[s])
    return y, last


def selective_scan_backward(x, dt, a, b, c, offsets, h0, skip, dt_bias, dy, dlast, backwards=False):
    """dict of dx, ddt, da, db, dc, dskip, ddt_bias, dh0"""
    v = dt + dt_bias
    d = softplus(v)
    before, after = np.zeros((len(x),) + a.shape), np.zeros((len(x),) + a.shape)

    def seen(t, s, i, p, q):
        before[t], after[t] = p, q

    selective_scan(x, dt, a, b, c, offsets, h0, skip, dt_bias, backwards, seen)
    out = {"dx": skip * dy, "ddt": np.zeros_like(dt), "da": np.zeros_like(a), "db": np.zeros_like(b), "dc": np.zeros_like(c),
           "dskip": (dy * x).sum(0), "dh0": dlast.copy()}
    for s in range(len(offsets) - 1):
        flow = dlast[s].copy()                                           # reaches the state after the row
        for t in reversed(_rows(offsets, s, backwards)):
            g = flow + dy[t][:, None] * c[t]
            keep = np.exp(d[t][:, None] * a)
            out["dc"][t] = dy[t] @ after[t]
            out["db"][t] = (d[t] * x[t]) @ g
            through, gb = g * keep * before[t], g @ b[t]
            out["da"] += through * d[t][:, None]
            out["dx"][t] += d[t] * gb
            out["ddt"][t] = ((through * a).sum(1) + gb * x[t]) * sigmoid(v[t])
            flow = keep * g
        out["dh0"][s] = flow
    out["ddt_bias"] = out["ddt"].sum(0)
    return out


def rms(v, eps):
    return v / np.sqrt((v * v).mean(1, keepdims=True) + eps)


def gated_residual(x, branch, gate, post, scale, following, eps):
    """(sum, y); gate may be None"""
    act = activate("silu", gate)[0] if gate is not None else 1.0
    total = x + scale * (act * rms(branch, eps) * post)
    return total, rms(total, eps) * following


def _rms_backward(v, eps, dh):
    """The gradient of v for that of its norm."""
    r = 1 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    return r * (dh - v * r * (dh * v * r).mean(1, keepdims=True))


def gated_residual_backward(x, branch, gate, post, scale, following, eps, dsum, dy):
    """dict of dx, dbranch, dgate, dpost, dscale, dnext"""
    act, slope = activate("silu", gate) if gate is not None else (np.ones_like(x), np.zeros_like(x))
    bh = rms(branch, eps)
    total = x + scale * (act * bh * post)
    ds = dsum + _rms_backward(total, eps, dy * following)
    return {"dx": ds, "dbranch": _rms_backward(branch, eps, ds * scale * act * post), "dgate": ds * scale * bh * post * slope,
            "dpost": scale * (ds * act * bh).sum(0), "dscale": (ds * act * bh * post).sum(keepdims=True).reshape(1), "dnext": (dy * rms(total, eps)).sum(0)}
