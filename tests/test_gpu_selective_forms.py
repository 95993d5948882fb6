"""The selective scan in every form that long lists walk in (states a lane, lanes a channel), which the rows and channels of a call choose: wide rows, of whose
channels the oracle follows some; the others have no part in the gradients that all share."""
import numpy as np
import pytest
import torch

from oracle import selective as V
from paper_2507_04123_amd import binding as B

import selective_bounds as L
from selective_helpers import DT, TYPES, draw, f64, offsets, rows, within, work

pytestmark = pytest.mark.gpu
WIDE = 2100


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


# Rows by states: up to 16 states in all three forms (2500, 2000 and 1000 rows), up to 8 in two, up to 32 in two, more in one; whole lanes and ragged ones.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,m", [(2500, 8), (2500, 5), (2000, 7), (2000, 8), (2500, 16), (2500, 11), (2000, 13), (2000, 16), (1000, 16), (1000, 9), (1300, 32), (1300, 20),
                                 (1000, 27), (1000, 32), (700, 64), (700, 3)])
def test_forms_of_long_lists(ctx, dtype, n, m):
    _check(ctx, dtype, [n // 3, 0, 1, 17, n - n // 3 - 18], WIDE, m, [0, 1, 5, 63, 64, 1030, 1031, 2047, 2048, 2096, 2098, 2099])


@pytest.mark.parametrize("dtype,lens,m", [("f16", [11, 0, 9], 64), ("bf16", [520, 20], 3)])
def test_as_many_channels_as_there_may_be(ctx, dtype, lens, m):
    _check(ctx, dtype, lens, 65536, m, [0, 7, 8, 4095, 32768, 65528, 65535])


def _check(ctx, dtype, lens, c, m, some):
    n, backwards = sum(lens), m % 2 == 1
    off, dev = offsets(lens)
    s = len(lens)
    p = {"x": draw(1, n, c, dtype=dtype), "dt": draw(2, n, c, scale=1.5, dtype=dtype), "b": draw(3, n, m, dtype=dtype), "c": draw(4, n, m, dtype=dtype),
         "a": -torch.exp(draw(5, c, m, scale=1.2)).float(), "skip": draw(6, c), "dt_bias": draw(7, c, shift=-3.0), "h0": draw(8, s, c, m)}
    dy, dlast = torch.zeros((n, c), dtype=p["x"].dtype), torch.zeros((s, c, m))
    dy[:, some], dlast[:, some] = draw(9, n, len(some), dtype=dtype), draw(10, s, len(some), m)
    g = {k: rows(t, "odd") if k in ("x", "dt", "b", "c") else t.cuda() for k, t in p.items()}
    args = [g[k] for k in ("x", "dt", "a", "b", "c")]
    scratch = work(ctx.selective_scan_work(DT[dtype], n, c, m))
    y, last = torch.full_like(dy, -3.0, device="cuda"), torch.full_like(dlast, -3.0, device="cuda")
    ctx.selective_scan(DT[dtype], *args, dev, y, scratch, skip=g["skip"], dt_bias=g["dt_bias"], backwards=backwards, h0=g["h0"], last=last)
    out = {k: torch.full_like(t, 9.0, device="cuda") for k, t in (("dx", dy), ("ddt", dy), ("db", p["b"]), ("dc", p["c"]), ("da", p["a"]), ("dskip", p["skip"]),
                                                                  ("ddt_bias", p["dt_bias"]), ("dh0", dlast))}
    ctx.selective_scan_backward(DT[dtype], *args, dev, dy.cuda(), *[out[k] for k in ("dx", "ddt", "da", "db", "dc")], scratch, skip=g["skip"], dskip=out["dskip"],
                                dt_bias=g["dt_bias"], ddt_bias=out["ddt_bias"], backwards=backwards, h0=g["h0"], dlast=dlast.cuda(), dh0=out["dh0"])
    e = {k: f64(t) for k, t in p.items()}
    mine = [e["x"][:, some], e["dt"][:, some], e["a"][some], e["b"], e["c"], off, e["h0"][:, some], e["skip"][some], e["dt_bias"][some]]
    ey, el = V.selective_scan(*mine, backwards)
    by, bl = L.selective_scan(*mine, backwards, dtype)
    within(y[:, some], ey, by, "y")
    within(last[:, some], el, bl, "last")
    mine += [f64(dy[:, some]), f64(dlast[:, some]), backwards]
    exp, bound = V.selective_scan_backward(*mine), L.selective_scan_backward(*mine, dtype)
    for k, t in out.items():
        t = t if k in ("db", "dc") else t[:, some] if k in ("dx", "ddt", "dh0") else t[some]
        within(t, exp[k], bound[k], k)
    others = np.setdiff1d(np.arange(c), some)
    assert torch.isfinite(y).all() and torch.isfinite(last).all() and not any(out[k][:, others].any() for k in ("dx", "ddt", "dh0"))
    assert not any(out[k][others].any() for k in ("da", "dskip", "ddt_bias"))
