"""An infinity or NaN in a recurrence stays in the state to the end of its sequence, wherever the kernels cut the rows and whatever the gates'
product has become by then, and reaches nothing else."""
import numpy as np
import pytest
import torch

from paper_2507_04123_amd import binding as B

pytestmark = pytest.mark.gpu

TD = {B.F32: torch.float32, B.F16: torch.float16, B.BF16: torch.bfloat16}
CHANNEL = 5
# sequences, channels, row of the fault: within one wave's rows; over blocks of one tile; over blocks of several tiles, the gates' product long 0
SIZES = {"short": ([9, 20, 3], 64, 13), "blocks": ([700, 0, 2200, 90], 64, 900), "tiles": ([1000, 0, 64000, 5000], 64, 21000),
         "odd": ([300, 4000, 1], 7, 1000)}


def _inputs(dtype, lens, c, seed):
    r = np.random.RandomState(seed)
    off, n = np.concatenate([[0], np.cumsum(lens)]), sum(lens)
    x, gate, dy = (torch.from_numpy(r.standard_normal((n, c)) * s + m).to(TD[dtype]) for s, m in ((1, 0), (2, 1.5), (1, 0)))
    gate[::41] = -300.0                                      # shut: the state is replaced
    h0, dlast = (torch.from_numpy(r.standard_normal((len(lens), c))).float() for _ in range(2))
    return off, x, gate, dy, h0, dlast


@pytest.mark.parametrize("dtype", list(TD))
@pytest.mark.parametrize("backwards", [False, True])
@pytest.mark.parametrize("size", list(SIZES))
def test_not_finite_to_the_end_of_the_sequence(dtype, backwards, size):
    lens, c, at = SIZES[size]
    off, x, gate, dy, h0, dlast = _inputs(dtype, lens, c, 7)
    s = int(np.searchsorted(off, at, "right")) - 1
    lo, hi = int(off[s]), int(off[s + 1])
    ctx = B.Context(1, 1, 1)
    offsets = torch.from_numpy(off.astype(np.int32)).cuda()
    work = torch.empty(max(16, ctx.recurrence_work(dtype, len(x), c)), dtype=torch.uint8, device="cuda")

    def run(x, gate, dy, h0, dlast):
        x, gate, dy, h0, dlast = (t.cuda() for t in (x, gate, dy, h0, dlast))
        y, last, dx, dgate, dh0 = torch.empty_like(x), torch.empty_like(h0), torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
        ctx.recurrence(dtype, x, gate, offsets, y, work, backwards=backwards, h0=h0, last=last)
        ctx.recurrence_backward(dtype, x, gate, offsets, dy, dx, dgate, work, backwards=backwards, h0=h0, dlast=dlast, dh0=dh0)
        return {"y": y, "last": last, "dx": dx, "dgate": dgate, "dh0": dh0}

    clean = run(x, gate, dy, h0, dlast)
    behind = slice(lo, at + 1) if backwards else slice(at, hi)       # the fault's row and those that the scan comes to after it
    before = slice(at, hi) if backwards else slice(lo, at + 1)
    rows, state = slice(lo, hi), slice(s, s + 1)
    # what is poisoned (its place), and the parts of the results that are not finite any more
    cases = {"x": (1, at, {"y": behind, "last": state}), "gate": (0, at, {"y": behind, "last": state, "dx": before, "dh0": state}),
             "dy": (0, at, {"dx": before, "dgate": before, "dh0": state}), "h0": (0, s, {"y": rows, "last": state}),
             "dlast": (0, s, {"dx": rows, "dgate": rows, "dh0": state})}
    for what, (with_inf, place, gone) in cases.items():
        for value in (float("nan"), float("inf")) if with_inf else (float("nan"),):
            args = {"x": x, "gate": gate, "dy": dy, "h0": h0, "dlast": dlast}
            args[what] = args[what].clone()
            args[what][place, CHANNEL] = value
            dirty = run(**args)
            for k, part in gone.items():
                bad = ~torch.isfinite(dirty[k][part, CHANNEL])
                assert bool(bad.all()), (what, value, k, int((~bad).sum()))
            for k, got in dirty.items():                             # everything outside of the sequence's channel is as it was, bit by bit
                same = torch.ones_like(got, dtype=torch.bool)
                same[state if k in ("last", "dh0") else rows, CHANNEL] = False
                assert torch.equal(torch.where(same, got, 0), torch.where(same, clean[k], 0)), (what, value, k)
    ctx.status_sync()
    ctx.close()
