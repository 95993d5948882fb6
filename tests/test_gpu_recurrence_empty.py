"""Many sequences, most of them without a row (streams that a sweep adds nothing to): their states are handed on, at the cost of a copy."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from paper_2507_04123_amd import binding as B

import sequence_bounds as L

pytestmark = pytest.mark.gpu

DT = {"f32": (B.F32, torch.float32), "f16": (B.F16, torch.float16)}


def _call(ctx, dtype, c, off, backwards=False, states=True):
    dt, td = DT[dtype]
    n, seqs, r = int(off[-1]), len(off) - 1, np.random.RandomState(c)
    x, gate, dy = (torch.from_numpy(r.standard_normal((n, c))).to(td).cuda() for _ in range(3))
    h0, dlast = (torch.from_numpy(r.standard_normal((seqs, c))).float().cuda() if states else None for _ in range(2))
    last, dh0 = (torch.full((seqs, c), 7.0, device="cuda") for _ in range(2))
    y, dx, dgate = (torch.full_like(x, 7.0) for _ in range(3))
    offsets = torch.from_numpy(np.asarray(off, dtype=np.int32)).cuda()
    work = torch.empty(max(16, ctx.recurrence_work(dt, n, c)), dtype=torch.uint8, device="cuda")

    def forward():
        ctx.recurrence(dt, x, gate, offsets, y, work, backwards=backwards, h0=h0, last=last)

    def gradients():
        ctx.recurrence_backward(dt, x, gate, offsets, dy, dx, dgate, work, backwards=backwards, h0=h0, dlast=dlast, dh0=dh0)

    return forward, gradients, (x, gate, h0, dy, dlast), (y, last, dx, dgate, dh0)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("c", [1, 3, 7, 64, 130])
@pytest.mark.parametrize("n,seqs", [(1, 1), (0, 70), (9, 1000), (900, 5000), (3000, 700)])
@pytest.mark.parametrize("states", [True, False])
def test_states_of_empty_sequences_are_handed_on(dtype, c, n, seqs, states):
    r = np.random.RandomState(seqs)
    off = np.concatenate([[0], np.sort(r.randint(0, n + 1, seqs - 1)), [n]])
    ctx = B.Context(1, 1, 1)
    for backwards in (False, True):
        forward, gradients, operands, results = _call(ctx, dtype, c, off, backwards, states)
        forward()
        gradients()
        x, gate, h0, dy, dlast = (np.zeros((seqs, c)) if t is None else t.double().cpu().numpy() for t in operands)
        exp = (*S.recurrence(x, gate, off, h0, backwards), *S.recurrence_backward(x, gate, off, h0, dy, dlast, backwards))
        bounds = (*L.recurrence(x, gate, off, h0, backwards, dtype)[:2], *L.recurrence_backward(x, gate, off, h0, dy, dlast, backwards, dtype))
        empty = off[1:] == off[:-1]
        for got, e, b, what in zip(results, exp, bounds, ("y", "last", "dx", "dgate", "dh0")):
            got = got.double().cpu().numpy()
            assert np.all(np.abs(got - e) <= b), what
            if what in ("last", "dh0"):
                assert np.array_equal(got[empty], e[empty]), what
    ctx.status_sync()
    ctx.close()


def test_empty_sequences_cost_a_copy():
    """4096 sequences with 8 rows in all: 2 MB of states to hand on.  200 us is over ten times what the launches and the copy take."""
    ctx = B.Context(1, 1, 1)
    off = np.sort(np.concatenate([[0], np.random.RandomState(1).randint(0, 9, 4095), [8]]))
    for call in _call(ctx, "f16", 128, off)[:2]:
        times = []
        for _ in range(12):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            call()
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b) * 1000)
        assert sorted(times)[6] < 200, times
    ctx.status_sync()
    ctx.close()
