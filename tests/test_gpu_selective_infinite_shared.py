"""The selective scan with an infinite value in B or C, which all channels share, where channels leave lanes of a wave without one."""
import numpy as np
import pytest

from oracle import selective as V
from paper_2507_04123_amd import binding as B

import selective_bounds as L
from selective_helpers import TYPES, offsets
from selective_infinite import GRADS, case, oracle, run, same_kind

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


# What the formula leaves finite does not depend on the value.  A single channel: sums over channels are infinite, not NaN.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [2, 4, 8, 13, 16, 32, 64])
@pytest.mark.parametrize("what", ["b", "c"])
def test_infinite_b_or_c(ctx, dtype, m, what):
    for lens in ([40, 30, 0, 20], [400, 600, 0, 60]):
        off, dev = offsets(lens)
        for c, at, backwards in ((1, 11, False), (1, 16, True), (37, 16, False)):
            p, row = case(lens, c, m, dtype), int(off[1]) + at
            args, grads = oracle(p, off, backwards)
            by, bl = L.selective_scan(*args, backwards, dtype)
            bound = L.selective_scan_backward(*grads, dtype)
            p[what][row, m // 2] = float("inf")
            y, last, out = run(ctx, dtype, p, dev, backwards)
            args, grads = oracle(p, off, backwards)
            with np.errstate(invalid="ignore"):
                ey, el = V.selective_scan(*args, backwards)
                exp = V.selective_scan_backward(*grads)
            if c == 1:
                hit = {"b": "dc", "c": "db"}[what]
                assert np.isinf(exp[hit][row, m // 2]) and not np.isnan(exp[hit]).any()
            same_kind(y, ey, by, "y")
            same_kind(last, el, bl, "last")
            for k in GRADS:
                same_kind(out[k], exp[k], bound[k], (k, c, at, backwards))
