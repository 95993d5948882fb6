"""The selective scan where channels leave lanes of a wave without one: those have no part in what all channels share, whatever channel 0 holds, and whatever
another block is writing there."""
import numpy as np
import pytest
import torch

from oracle import selective as V
from paper_2507_04123_amd import binding as B

import selective_bounds as L
from selective_helpers import TYPES, offsets, work
from selective_infinite import GRADS, case, oracle, run, same_kind

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


# An infinite value or step in one row of channel 0.  What the formula leaves finite does not depend on the value, nor on a step beyond some thousands, whose decays
# are 0: the bounds are taken from such a call.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [[40, 30, 0, 20], [400, 600, 0, 60]])
@pytest.mark.parametrize("what,finite", [("x", 1.0), ("dt", 30000.0)])
def test_infinite_rows_of_channel_0(ctx, dtype, lens, what, finite):
    off, dev = offsets(lens)
    for c, m, at, backwards in ((9, 16, 11, False), (9, 16, 16, True), (5, 4, 8, False), (70, 32, 21, False)):
        p = case(lens, c, m, dtype)
        row = int(off[1]) + at
        p["x"][row, 0] = 2.0
        p[what][row, 0] = finite
        args, grads = oracle(p, off, backwards)
        by, bl = L.selective_scan(*args, backwards, dtype)
        bound = L.selective_scan_backward(*grads, dtype)
        p[what][row, 0] = float("inf")
        y, last, out = run(ctx, dtype, p, dev, backwards)
        args, grads = oracle(p, off, backwards)
        with np.errstate(invalid="ignore"):
            ey, el = V.selective_scan(*args, backwards)
            exp = V.selective_scan_backward(*grads)
        same_kind(y, ey, by, "y")
        same_kind(last, el, bl, "last")
        for k in GRADS:
            same_kind(out[k], exp[k], bound[k], (k, c, m))
        assert np.isinf(exp["db"][row]).all() and np.isfinite(np.delete(exp["db"], row, 0)).all() and np.isinf(ey[row, 0])


# More channels than a block has lanes for, so that blocks side by side share the sums, and lanes without a channel in the last one; results in place, and infinite ones
# in channel 0's.
@pytest.mark.parametrize("c,m,lens", [(265, 16, [300, 0, 211]), (290, 16, [40, 33]), (265, 16, [21000]), (45, 64, [100, 77]), (300, 30, [500])])
def test_results_in_place_of_several_blocks(ctx, c, m, lens):
    off, dev = offsets(lens)
    p = case(lens, c, m, "f16")
    p["skip"][0] = 1e6                                                       # channel 0: dx and y beyond the type's range
    y, last, want = run(ctx, "f16", p, dev, False)
    assert torch.isinf(want["dx"][:, 0]).any() and torch.isinf(y[:, 0]).any()
    assert all(torch.isfinite(want[k]).all() for k in GRADS[1:]) and torch.isfinite(want["dx"][:, 1:]).all() and torch.isfinite(y[:, 1:]).all()
    g = {k: t.cuda() for k, t in p.items()}
    w = work(ctx.selective_scan_work(B.F16, len(y), c, m))
    kw = dict(skip=g["skip"], dt_bias=g["dt_bias"], h0=g["h0"])
    for _ in range(3):
        x, dt = g["x"].clone(), g["dt"].clone()
        out = {k: torch.empty_like(want[k]) for k in GRADS[2:]}
        ctx.selective_scan_backward(B.F16, x, dt, g["a"], g["b"], g["c"], dev, g["dy"], x, dt, out["da"], out["db"], out["dc"], w, dskip=out["dskip"],
                                    ddt_bias=out["ddt_bias"], dlast=g["dlast"], dh0=out["dh0"], **kw)
        out.update(dx=x, ddt=dt)
        for k in GRADS:
            assert torch.equal(out[k], want[k]), k
        x, end = g["x"].clone(), torch.empty_like(last)
        ctx.selective_scan(B.F16, x, g["dt"], g["a"], g["b"], g["c"], dev, x, w, last=end, **kw)
        assert torch.equal(x, y) and torch.equal(end, last)
