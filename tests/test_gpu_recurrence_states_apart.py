"""The recurrence's last states must not lie on its first ones, nor the gradient of the first on that of the last: other waves may still
have to read what one has written.  Such calls are refused before anything is launched."""
import pytest
import torch

from paper_2507_04123_amd import binding as B

pytestmark = pytest.mark.gpu


def test_states_that_overlap_are_refused():
    ctx, c, n, seqs = B.Context(1, 1, 1), 8, 20, 3
    x, gate, dy = (torch.randn(n, c, device="cuda") for _ in range(3))
    offsets = torch.tensor([0, 7, 7, n], dtype=torch.int32, device="cuda")
    work = torch.empty(max(16, ctx.recurrence_work(B.F32, n, c)), dtype=torch.uint8, device="cuda")
    states = torch.randn(2 * seqs, c, device="cuda")
    before, y, dgate = states.clone(), torch.full_like(x, 3.0), torch.full_like(x, 3.0)
    for at in (0, 1, seqs - 1):                              # the same place, and any overlap
        for p, q in ((states[:seqs], states[at:at + seqs]), (states[at:at + seqs], states[:seqs])):
            with pytest.raises(B.Emc2Error, match="overlap") as ei:
                ctx.recurrence(B.F32, x, gate, offsets, y, work, h0=p, last=q)
            assert ei.value.status == B.ERR_INVALID_ARG
            with pytest.raises(B.Emc2Error, match="overlap"):
                ctx.recurrence_backward(B.F32, x, gate, offsets, dy, y, dgate, work, dlast=p, dh0=q)
    torch.cuda.synchronize()
    assert torch.equal(states, before) and bool((y == 3.0).all())
    one, two, last = states[:seqs], states[seqs:], torch.empty(seqs, c, device="cuda")
    ctx.recurrence(B.F32, x, gate, offsets, y, work, h0=one.clone(), last=last)
    ctx.recurrence(B.F32, x, gate, offsets, y, work, h0=one, last=two)                    # neighbours are apart
    assert torch.equal(two, last)
    exp = torch.empty_like(last)
    ctx.recurrence_backward(B.F32, x, gate, offsets, dy, torch.empty_like(x), dgate, work, h0=one.clone(), dlast=two, dh0=exp)
    ctx.recurrence_backward(B.F32, x, gate, offsets, dy, torch.empty_like(x), dgate, work, h0=one, dlast=two, dh0=one)   # on the first states: allowed
    assert torch.equal(one, exp)
    ctx.status_sync()
    ctx.close()
