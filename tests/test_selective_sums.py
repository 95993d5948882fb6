"""The bounds that the parameters' gradients of long scans are held to (CPU): a sum that has lost a chunk of rows, or all, falls outside."""
import numpy as np
import pytest

from oracle import selective as V

import selective_sums as S
from selective_helpers import f64

NAMES = ("x", "dt", "a", "b", "c", "h0", "skip", "dt_bias", "dy", "dlast")


@pytest.mark.parametrize("backwards", [False, True])
def test_a_lost_chunk_is_outside(backwards):
    e = {k: f64(t) for k, t in S.case("f16").items()}
    off = np.concatenate([[0], np.cumsum(S.LENS)])
    args = [e[k] for k in NAMES[:5]] + [off] + [e[k] for k in NAMES[5:]] + [backwards]
    terms, bounds = S.terms_and_bounds(*args)
    exact = V.selective_scan_backward(*args)
    n, chunk = len(e["x"]), S.chunk_rows(len(e["x"]))
    for k in S.NAMES:
        walk = terms[k][::-1] if backwards else terms[k]
        assert np.allclose(walk.sum(0), exact[k], rtol=1e-10, atol=0)
        assert (bounds[k] < 0.001 * np.abs(exact[k])).all()
        chunks = np.add.reduceat(walk, range(0, n - n % chunk, chunk))
        assert (np.abs(chunks) > bounds[k]).mean() > 0.99, (k, float(bounds[k].max()), float(np.abs(chunks).min()))
