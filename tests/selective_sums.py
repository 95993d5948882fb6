"""Sums over the rows of long calls of the selective scan, the gradients of its parameters: cases whose rows add to them with one sign, so that losing a few
of the rows shows, and how far the sums may be off."""
import numpy as np
import torch

from oracle.sequence import _rows, sigmoid

import selective_bounds as L
from selective_helpers import draw

E = L.E
LENS = [17000, 0, 5, 1, 130, 2048, 0, 0, 3, 24000, 16, 15, 8, 26774]
NAMES = ("da", "dskip", "ddt_bias")


def case(dtype, c=3, m=3):
    """70 000 rows: positive x, B, C and dy, states that remember some rows."""
    n, s = sum(LENS), len(LENS)
    p = {k: draw(i, n, w, dtype=dtype).abs() + 0.25 for i, (k, w) in enumerate((("x", c), ("b", m), ("c", m), ("dy", c)))}
    p.update(dt=draw(5, n, c, scale=0.5, dtype=dtype), a=-torch.exp(draw(6, c, m, scale=0.3)), dt_bias=torch.full((c,), 0.5), skip=draw(7, c).abs(),
             h0=torch.zeros(s, c, m), dlast=torch.zeros(s, c, m))
    return p


def chunk_rows(n):
    """Rows that a thread adds one after the other: a call of one slice of channels is cut into 2048 chunks of whole batches of eight rows, of 16 rows at least."""
    return max(16, -(-(-(-n // 2048)) // 8) * 8)


def behind(n):
    """Additions behind a row's part at most: those of its chunk; one for every 256 chunks; eight for these by halves; four for lanes that share rows."""
    chunk = chunk_rows(n)
    return chunk + -(-(-(-n // chunk)) // 256) + 8 + 4


def terms_and_bounds(x, dt, a, b, c, off, h0, skip, dt_bias, dy, dlast, backwards):
    """(what every row adds, bounds of the sums): the rows' own bounds are those of selective_bounds, the sum's `behind` roundings of every part."""
    v, d, ed = L._steps(x, dt, a, dt_bias)
    before, after, eb, ea, _ = L._scan_states(x, dt, a, b, c, off, h0, dt_bias, backwards)
    k, kn = (16 + a.shape[1]) * E, behind(len(x)) * E
    terms = {"da": np.zeros((len(x),) + a.shape), "dskip": dy * x, "ddt_bias": np.zeros_like(x)}
    bounds = {"da": np.zeros_like(a), "dskip": ((kn + E) * np.abs(dy * x)).sum(0), "ddt_bias": np.zeros_like(skip)}
    for s in range(len(off) - 1):
        flow, err = dlast[s].copy(), np.zeros(a.shape)
        for t in reversed(_rows(off, s, backwards)):
            own = dy[t][:, None] * c[t]
            g, eg = flow + own, err + 4 * E * (np.abs(flow) + np.abs(own))
            keep, rel = L._decay(d[t], ed[t], a)
            gb, egb = g @ b[t], (eg + k * np.abs(g)) @ np.abs(b[t])
            through = g * keep * before[t]
            eth = keep * (eg * np.abs(before[t]) + np.abs(g) * (rel * np.abs(before[t]) + eb[t])) + 4 * E * np.abs(through)
            dd = (through * a).sum(1) + gb * x[t]
            edd = ((eth + k * np.abs(through)) * np.abs(a)).sum(1) + egb * np.abs(x[t]) + 4 * E * np.abs(gb * x[t])
            on = sigmoid(v[t])
            terms["da"][t], terms["ddt_bias"][t] = through * d[t][:, None], dd * on
            bounds["da"] += (eth + kn * np.abs(through)) * d[t][:, None] + np.abs(through) * ed[t][:, None]
            bounds["ddt_bias"] += on * (edd + (16 + 2 * np.abs(v[t])) * E * np.abs(dd)) + kn * np.abs(dd * on)
            flow, err = keep * g, keep * (eg + (rel + 4 * E) * np.abs(g)) + L.TINY["f32"]
    return terms, bounds
