"""How far a result of the selective state space operators may be from the oracle's, element by element, from the number formats alone; written like
the bounds of the sequence operators, whose constants it takes: an fp32 sum of magnitudes that add up to s, with at most k additions in a row behind each
term, is within k E s, a rounding to a type within U of the value."""
from __future__ import annotations

import numpy as np

from oracle import selective as V
from oracle.sequence import _rows, activate, sigmoid

from sequence_bounds import E, K, TINY, U, rounded  # noqa: F401


def _silu(z, ez):
    """silu of z and its slope, and their bounds: the exponential is exact to E |z|, the slope of silu below 1.1, that of its slope at most 0.5."""
    value, slope = activate("silu", z)
    return value, slope, 1.1 * ez + 16 * E * (1 + np.abs(z)) * np.abs(value) + TINY["f32"], 0.5 * ez + 32 * E * (1 + np.abs(z) ** 2) * (np.abs(slope) + 0.01)


def _conv_rows(x, w, bias, off, before, silu, backwards, dtype, dy=None, dlast=None):
    """Per row: bounds of y; with dy also those of dx, dw, dbias and dbefore."""
    taps, n = len(w), len(x)
    by = np.zeros_like(x)
    dx, dxb, dw, db = np.zeros_like(x), np.zeros_like(x), np.zeros_like(w), np.zeros_like(bias)
    dbefore = np.zeros_like(before)
    chain = (64 + n / 8) * E                 # of a weight's sum: rows of a thread, runs of a block, blocks by halves; runs have eight rows at least
    for s in range(len(off) - 1):
        rows = _rows(off, s, backwards)
        flow, size = (np.zeros((taps - 1 + len(rows), x.shape[1])) for _ in range(2))
        for i, t in enumerate(rows):
            past = [V._history(x, before, rows, i, k, s) for k in range(taps)]
            z = bias + sum(w[k] * past[k] for k in range(taps))
            ez = (taps + 4) * E * (np.abs(bias) + sum(np.abs(w[k] * past[k]) for k in range(taps)))
            value, slope, ev, es = _silu(z, ez) if silu else (z, np.ones_like(z), ez, np.zeros_like(z))
            by[t] = rounded(value, ev, dtype)
            if dy is None:
                continue
            dz = dy[t] * slope
            edz = np.abs(dy[t]) * es + 2 * E * np.abs(dz)
            db += edz + chain * np.abs(dz)
            for k in range(taps):
                dw[k] += (edz + chain * np.abs(dz)) * np.abs(past[k])
                flow[taps - 1 + i - k] += np.abs(w[k]) * (edz + (taps + 4) * E * np.abs(dz))
                size[taps - 1 + i - k] += w[k] * dz
        if dy is not None:
            flow[len(rows):] += (taps + 4) * E * np.abs(dlast[s])
            size[len(rows):] += dlast[s]
            dbefore[s] = flow[:taps - 1]
            if rows:
                dxb[rows], dx[rows] = flow[taps - 1:], size[taps - 1:]
    if dy is None:
        return by
    t = TINY["f32"]
    return rounded(dx, dxb, dtype), dw + t, db + t, dbefore + t


def causal_conv(x, w, bias, off, before, silu, backwards, dtype):
    return _conv_rows(x, w, bias, off, before, silu, backwards, dtype)


def causal_conv_backward(x, w, bias, off, before, dy, dlast, silu, backwards, dtype):
    return _conv_rows(x, w, bias, off, before, silu, backwards, dtype, dy, dlast)


def _steps(x, dt, a, dt_bias):
    """The steps and their bounds; the relative bound of a row's decay is _decay of them.  v = dt + bias is rounded once, which moves the step by E |v| of itself at
    most, and so does the exponential in it; the logarithm is good to a few units."""
    v = dt + dt_bias
    d = V.softplus(v)
    return v, d, (16 + 2 * np.abs(v)) * E * d + TINY["f32"]


def _decay(d, ed, a):
    """A row's decays and their relative bounds.  K also covers that a run of rows is one exponential of the summed steps: as many additions behind each."""
    keep = np.exp(d[:, None] * a)
    return keep, np.abs(a) * ed[:, None] + (K + 4 * np.abs(d[:, None] * a)) * E


def _scan_states(x, dt, a, b, c, off, h0, dt_bias, backwards):
    """For every row the state before and after it and their bounds, and the bound of every sequence's last."""
    _, d, ed = _steps(x, dt, a, dt_bias)
    shape = (len(x),) + a.shape
    before, after, eb, ea = (np.zeros(shape) for _ in range(4))
    last = np.zeros_like(h0)
    for s in range(len(off) - 1):
        h, err = h0[s], np.zeros(a.shape)
        for t in _rows(off, s, backwards):
            before[t], eb[t] = h, err
            keep, rel = _decay(d[t], ed[t], a)
            gain = d[t] * x[t]
            add = gain[:, None] * b[t]
            err = keep * (err + rel * np.abs(h)) + (ed[t] * np.abs(x[t]))[:, None] * np.abs(b[t]) + 8 * E * (keep * np.abs(h) + np.abs(add)) + TINY["f32"]
            h = keep * h + add
            after[t], ea[t] = h, err
        last[s] = err
    return before, after, eb, ea, last


def selective_scan(x, dt, a, b, c, off, h0, skip, dt_bias, backwards, dtype):
    """Bounds of (y, last)."""
    _, after, _, ea, last = _scan_states(x, dt, a, b, c, off, h0, dt_bias, backwards)
    k = (16 + a.shape[1]) * E
    y = np.einsum("tcn,tn->tc", after, c) + skip * x
    ey = np.einsum("tcn,tn->tc", ea + k * np.abs(after), np.abs(c)) + k * np.abs(skip * x)
    return rounded(y, ey, dtype), last + TINY["f32"]


def selective_scan_backward(x, dt, a, b, c, off, h0, skip, dt_bias, dy, dlast, backwards, dtype):
    """dict of the gradients' bounds"""
    v, d, ed = _steps(x, dt, a, dt_bias)
    before, after, eb, ea, _ = _scan_states(x, dt, a, b, c, off, h0, dt_bias, backwards)
    exact = V.selective_scan_backward(x, dt, a, b, c, off, h0, skip, dt_bias, dy, dlast, backwards)
    k, kc, kn = (16 + a.shape[1]) * E, (16 + x.shape[1]) * E, (64 + len(x)) * E
    out = {name: np.zeros_like(t) for name, t in exact.items()}
    for s in range(len(off) - 1):
        flow, err = dlast[s].copy(), np.zeros(a.shape)
        for t in reversed(_rows(off, s, backwards)):
            gain, own = d[t] * x[t], dy[t][:, None] * c[t]
            egain = ed[t] * np.abs(x[t]) + 2 * E * np.abs(gain)
            g, eg = flow + own, err + 4 * E * (np.abs(flow) + np.abs(own))
            keep, rel = _decay(d[t], ed[t], a)
            out["dc"][t] = np.abs(dy[t]) @ (ea[t] + kc * np.abs(after[t]))
            out["db"][t] = np.abs(gain) @ (eg + kc * np.abs(g)) + egain @ np.abs(g)
            gb, egb = g @ b[t], (eg + k * np.abs(g)) @ np.abs(b[t])
            out["dx"][t] = d[t] * egb + ed[t] * np.abs(gb) + 4 * E * (np.abs(skip * dy[t]) + np.abs(d[t] * gb))
            through = g * keep * before[t]
            eth = keep * (eg * np.abs(before[t]) + np.abs(g) * (rel * np.abs(before[t]) + eb[t])) + 4 * E * np.abs(through)
            dd = (through * a).sum(1) + gb * x[t]
            edd = ((eth + k * np.abs(through)) * np.abs(a)).sum(1) + egb * np.abs(x[t]) + 4 * E * np.abs(gb * x[t])
            on = sigmoid(v[t])
            out["ddt"][t] = on * (edd + (16 + 2 * np.abs(v[t])) * E * np.abs(dd))
            out["da"] += (eth + kn * np.abs(through)) * d[t][:, None] + np.abs(through) * ed[t][:, None]
            out["ddt_bias"] += out["ddt"][t] + kn * np.abs(dd * on)
            out["dskip"] += kn * np.abs(dy[t] * x[t])
            flow, err = keep * g, keep * (eg + (rel + 4 * E) * np.abs(g)) + TINY["f32"]
        out["dh0"][s] = err
    for name in ("dx", "ddt", "db", "dc"):
        out[name] = rounded(exact[name], out[name], dtype)
    return {name: t + TINY["f32"] for name, t in out.items()}


def _join(x, branch, gate, post, scale, eps):
    m = lambda t: t.mean(1, keepdims=True)  # noqa: E731
    rb = 1 / np.sqrt(m(branch * branch) + eps)
    bh = branch * rb
    ebh = K * E * np.abs(bh)                                             # a sum of squares loses nothing
    act, slope, ea, es = _silu(gate, np.zeros_like(gate)) if gate is not None else (np.ones_like(x), np.zeros_like(x), np.zeros_like(x), np.zeros_like(x))
    t = scale * post * bh * act
    et = np.abs(scale * post) * (ebh * np.abs(act) + np.abs(bh) * ea) + 8 * E * np.abs(t)
    total = x + t
    etotal = et + 2 * E * (np.abs(x) + np.abs(t))
    rs = 1 / np.sqrt(m(total * total) + eps)
    rel = m(np.abs(total) * etotal) * rs * rs + K * E                    # of rs
    return dict(m=m, rb=rb, bh=bh, ebh=ebh, act=act, slope=slope, ea=ea, es=es, total=total, etotal=etotal, rs=rs, rel=rel)


def gated_residual(x, branch, gate, post, scale, following, eps, dtype):
    """Bounds of (sum, y)."""
    j = _join(x, branch, gate, post, scale, eps)
    y = j["total"] * j["rs"] * following
    return (rounded(j["total"], j["etotal"], dtype),
            rounded(y, np.abs(following) * j["rs"] * (j["etotal"] + np.abs(j["total"]) * (j["rel"] + 4 * E)), dtype))


def gated_residual_backward(x, branch, gate, post, scale, following, eps, dsum, dy, dtype):
    j = _join(x, branch, gate, post, scale, eps)
    m, rb, bh, ebh, act, slope, ea, es, rs, rel = (j[k] for k in ("m", "rb", "bh", "ebh", "act", "slope", "ea", "es", "rs", "rel"))
    A = np.abs
    exact = V.gated_residual_backward(x, branch, gate, post, scale, following, eps, dsum, dy)
    th = j["total"] * rs
    eth = rs * j["etotal"] + A(th) * rel
    q = dy * following
    mean = m(q * th)
    emean = m(A(q) * eth) + K * E * m(A(q * th))
    eS = rs * ((rel + 6 * E) * (A(q) + A(th * mean)) + eth * A(mean) + A(th) * emean) + 4 * E * (A(dsum) + rs * (A(q) + A(th * mean)))
    S = exact["dx"]
    f = A(scale * post)
    d = S * scale * post * act
    e_d = f * (eS * A(act) + A(S) * ea) + 6 * E * A(d)
    mean_d = m(d * bh)
    emean_d = m(e_d * A(bh) + A(d) * ebh) + K * E * m(A(d * bh))
    col = eS * A(act * bh) + A(S) * (ea * A(bh) + A(act) * ebh)
    size = A(S * act * bh)
    rows = (64 + len(x) ** 0.5) * E
    out = {"dx": rounded(S, eS, dtype),
           "dbranch": rounded(exact["dbranch"], rb * (K * E * (A(d) + A(bh * mean_d)) + e_d + ebh * A(mean_d) + A(bh) * emean_d), dtype),
           "dgate": rounded(exact["dgate"], f * (eS * A(bh * slope) + A(S) * (ebh * A(slope) + A(bh) * es)) + 8 * E * A(exact["dgate"]), dtype),
           "dpost": A(scale) * (col + rows * size).sum(0) + TINY["f32"],
           "dscale": ((col + (rows + 16 * E) * size) * A(post)).sum().reshape(1) + TINY["f32"],
           "dnext": (A(dy) * eth + rows * A(dy * th)).sum(0) + TINY["f32"]}
    return out
