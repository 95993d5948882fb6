"""What the tests of infinite rows of the selective scan share: cases whose states remember hundreds of rows, all results of a call, and comparisons of values that
may be infinite or NaN."""
import numpy as np
import torch

from selective_helpers import DT, draw, f64, work

GRADS = ("dx", "ddt", "da", "db", "dc", "dskip", "ddt_bias", "dh0")


def case(lens, c, m, dtype):
    """States that remember hundreds of rows, B and C above 0: an infinite state has one sign."""
    n, s = sum(lens), len(lens)
    p = {"x": draw(1, n, c, dtype=dtype), "dt": draw(2, n, c, scale=0.5, dtype=dtype), "b": draw(3, n, m, dtype=dtype).abs() + 0.25,
         "c": draw(4, n, m, dtype=dtype).abs() + 0.25, "dy": draw(5, n, c, dtype=dtype), "a": -torch.exp(draw(6, c, m, scale=0.5, shift=-3.0)).float(),
         "skip": draw(7, c), "dt_bias": torch.full((c,), -4.0), "h0": draw(8, s, c, m), "dlast": draw(9, s, c, m)}
    return p


def run(ctx, dtype, p, dev, backwards):
    """(y, last, gradients), nothing in place."""
    g = {k: t.cuda() for k, t in p.items()}
    n, c = g["x"].shape
    w = work(ctx.selective_scan_work(DT[dtype], n, c, g["a"].shape[1]))
    args = [g[k] for k in ("x", "dt", "a", "b", "c")]
    kw = dict(skip=g["skip"], dt_bias=g["dt_bias"], backwards=backwards, h0=g["h0"])
    y, last = torch.empty_like(g["x"]), torch.empty_like(g["h0"])
    ctx.selective_scan(DT[dtype], *args, dev, y, w, last=last, **kw)
    out = {k: torch.empty_like(g[q]) for k, q in zip(GRADS, ("x", "dt", "a", "b", "c", "skip", "dt_bias", "h0"))}
    ctx.selective_scan_backward(DT[dtype], *args, dev, g["dy"], *[out[k] for k in ("dx", "ddt", "da", "db", "dc")], w, dskip=out["dskip"],
                                ddt_bias=out["ddt_bias"], dlast=g["dlast"], dh0=out["dh0"], **kw)
    return y, last, out


def oracle(p, off, backwards):
    e = {k: f64(t) for k, t in p.items()}
    args = [e[k] for k in ("x", "dt", "a", "b", "c")] + [off] + [e[k] for k in ("h0", "skip", "dt_bias")]
    return args, args + [e["dy"], e["dlast"], backwards]


def same_kind(got, exp, bound, what):
    """NaN where the formula gives NaN, an infinity where it gives that one; the finite values within the bound."""
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(exp)), what
    inf = np.isinf(exp)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], exp[inf]), what
    ok = np.isfinite(exp)
    assert (np.abs(got[ok] - exp[ok]) <= bound[ok]).all(), what
