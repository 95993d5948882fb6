"""The selective scan with an infinite step in one row, where the lanes of a channel have states that are none: what came before the row is forgotten, y behind it is
infinite, the gradients in front of it are finite; the same row by row."""
import numpy as np
import pytest
import torch

from oracle import selective as V
from paper_2507_04123_amd import binding as B

import selective_bounds as L
from selective_helpers import DT, TYPES, f64, offsets
from selective_infinite import GRADS, case, oracle, run, same_kind

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


# The bounds are those of a step of some thousands, whose decays are 0 as well.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 3, 7, 8, 12, 13, 16, 20, 33])
@pytest.mark.parametrize("lens", [[40, 30, 0, 20], [400, 600, 0, 60]])
def test_an_infinite_step_gives_what_the_formula_gives(ctx, dtype, m, lens):
    off, dev = offsets(lens)
    for at, backwards in ((16, False), (11, False), (16, True)):         # the first of eight rows that are walked together, and another
        p, row = case(lens, 9, m, dtype), int(off[1]) + at
        p["x"][row, 2] = 2.0
        p["dt"][row, 2] = 30000.0
        args, grads = oracle(p, off, backwards)
        by, bl = L.selective_scan(*args, backwards, dtype)
        bound = L.selective_scan_backward(*grads, dtype)
        p["dt"][row, 2] = float("inf")
        y, last, out = run(ctx, dtype, p, dev, backwards)
        args, grads = oracle(p, off, backwards)
        with np.errstate(invalid="ignore"):
            ey, el = V.selective_scan(*args, backwards)
            exp = V.selective_scan_backward(*grads)
        assert np.isposinf(ey[row, 2]) and np.isfinite(exp["dx"][:row]).all() and np.isfinite(np.delete(exp["db"], row, 0)).all()
        same_kind(y, ey, by, "y")
        same_kind(last, el, bl, "last")
        for k in GRADS:
            same_kind(out[k], exp[k], bound[k], (k, at, backwards))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [3, 12, 16, 20])
def test_row_by_row_it_is_the_same(ctx, dtype, m):
    n, at = 14, 5
    off, dev = offsets([n])
    p = case([n], 9, m, dtype)
    p["x"][at, 2], p["dt"][at, 2] = 2.0, 30000.0
    args, _ = oracle(p, off, False)
    by, bl = L.selective_scan(*args, False, dtype)
    p["dt"][at, 2] = float("inf")
    y, last, _ = run(ctx, dtype, p, dev, False)
    args, _ = oracle(p, off, False)
    ey, el = V.selective_scan(*args, False)
    g = {k: t.cuda() for k, t in p.items()}
    h, rows = g["h0"].clone(), torch.empty_like(y)
    for t in range(n):
        ctx.selective_scan_step(DT[dtype], *[g[k][t:t + 1] if k != "a" else g[k] for k in ("x", "dt", "a", "b", "c")], h, h, rows[t:t + 1], skip=g["skip"],
                                dt_bias=g["dt_bias"])
    for got in ((y, last), (rows, h)):
        same_kind(got[0], ey, by, "y")
        same_kind(got[1], el, bl, "last")
    assert np.isposinf(f64(rows[at:, 2])).all()
