"""Calls of a sequence block in other orders than run, backward."""
import numpy as np
import pytest
import torch

from paper_2507_04123_amd import binding as B
from paper_2507_04123_amd import gen
from paper_2507_04123_amd.sequence import SequenceBlock, sequence_params

pytestmark = pytest.mark.gpu

TD = {B.F32: torch.float32, B.F16: torch.float16, B.BF16: torch.bfloat16}


def _block(ctx, dtype, cap, frames, c, f, **more):
    return SequenceBlock(ctx, dtype, cap, frames, sequence_params(gen.make_sequence_params(c, f, 5), dtype), **more)


def _normal(seed, shape, dtype=torch.float32):
    return torch.from_numpy(np.random.RandomState(seed).standard_normal(shape)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [B.F32, B.F16, B.BF16])
def test_a_step_between_run_and_backward_changes_no_gradient(dtype):
    c, lens = 48, [30, 0, 1, 200]
    ctx = B.Context(1, 1, 1)
    b = _block(ctx, dtype, 240, 4, c, 64, train=True)
    x, dy, rows = _normal(1, (231, c), TD[dtype]), _normal(2, (231, c), TD[dtype]), _normal(3, (4, c), TD[dtype])
    offsets = torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device="cuda")
    h0, h = _normal(4, (4, c)), _normal(5, (4, c))

    def gradients(step):
        b.run(x, offsets, h0)
        if step:
            b.step(rows, h.clone())
        return [t.clone() for t in (b.backward(x, offsets, dy, h0), b.dh0, *b.grads.values())]

    plain = gradients(False)
    assert all(torch.equal(p, q) for p, q in zip(plain, gradients(True)))
    # and the step of a training block is that of one for serving
    serve = _block(ctx, dtype, 4, 4, c, 64)
    one, two = h.clone(), h.clone()
    assert torch.equal(b.step(rows, one), serve.step(rows, two)) and torch.equal(one, two) and not torch.equal(one, h)
    ctx.status_sync()
    ctx.close()


def test_parameters_of_other_shapes_are_refused():
    """The fragments' buffer would take smaller weights, which the block would then read as its own."""
    ctx = B.Context(1, 1, 1)
    b = _block(ctx, B.F16, 16, 1, 32, 96)
    x, offsets = _normal(1, (16, 32), torch.float16), torch.tensor([0, 16], dtype=torch.int32, device="cuda")
    before = b.run(x, offsets).clone()
    for c, f in ((32, 64), (16, 96), (32, 128)):
        with pytest.raises(ValueError, match="load"):
            b.load(sequence_params(gen.make_sequence_params(c, f, 6), B.F16))
    with pytest.raises(ValueError, match="load"):
        b.load({k: t for k, t in b.params.items() if k != "beta"})
    with pytest.raises(ValueError, match="wg"):
        b.load(sequence_params(gen.make_sequence_params(32, 96, 6), B.F32))
    assert torch.equal(b.run(x, offsets), before)             # the old ones are still there
    b.load(sequence_params(gen.make_sequence_params(32, 96, 6), B.F16))
    assert not torch.equal(b.run(x, offsets), before)
    ctx.status_sync()
    ctx.close()
