"""Capacities up to the 2^30 rows that the sequence operators accept: one launch holds the blocks of them all.  Rows beyond the device's count
are neither read nor written, so the buffers here are those of the rows present."""
import numpy as np
import pytest
import torch

from paper_2507_04123_amd import binding as B

import sequence_bounds as L

pytestmark = pytest.mark.gpu

TD = {B.F32: torch.float32, B.F16: torch.float16}
N = 77


@pytest.fixture
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


def _normal(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("dtype,c,capacity", [(B.F16, 128, 1 << 30), (B.F16, 200, 1 << 30), (B.F16, 512, 1 << 28), (B.F32, 1024, 1 << 27), (B.F32, 5, 1 << 30)])
def test_layernorm_of_a_large_capacity(ctx, dtype, c, capacity):
    td, st = TD[dtype], torch.cuda.current_stream().cuda_stream
    x, gamma, beta, count = _normal(1, N, c, dtype=td), _normal(2, c), _normal(3, c), torch.tensor([N], dtype=torch.int32, device="cuda")
    out = []
    for cap in (N, capacity):
        y = torch.empty_like(x)
        assert ctx.lib.emc2_layernorm(ctx.h, dtype, x.data_ptr(), c, None, 0, gamma.data_ptr(), beta.data_ptr(), 1e-5, count.data_ptr(), cap, c,
                                      None, 0, y.data_ptr(), c, st) == B.OK
        out.append(y)
    assert torch.equal(*out)


@pytest.mark.parametrize("c", [96, 130, 256])
def test_fp32_networks_of_a_large_capacity(ctx, c):
    f, capacity, st = 40, 1 << 28, torch.cuda.current_stream().cuda_stream
    x, dy, count = _normal(1, N, c), _normal(2, N, c), torch.tensor([N], dtype=torch.int32, device="cuda")
    w = [_normal(3 + i, *s) for i, s in enumerate(((c, f), (c, f), (f, c)))]
    packed = torch.empty(ctx.ffn_packed_size(B.F32, c, f), device="cuda")
    ctx.ffn_pack(B.F32, *w, packed)
    work = torch.empty(ctx.ffn_work(B.F32, capacity, c, f), dtype=torch.uint8, device="cuda")
    out = []
    for cap in (N, capacity):
        y, dx, g = torch.empty_like(x), torch.empty_like(x), [torch.empty_like(t) for t in w]
        assert ctx.lib.emc2_ffn(ctx.h, B.F32, B.ACT_SILU, x.data_ptr(), c, packed.data_ptr(), None, 0, count.data_ptr(), cap, c, f, y.data_ptr(),
                                c, st) == B.OK
        assert ctx.lib.emc2_ffn_backward(ctx.h, B.F32, B.ACT_SILU, x.data_ptr(), c, packed.data_ptr(), dy.data_ptr(), c, count.data_ptr(), cap, c,
                                         f, dx.data_ptr(), c, *(t.data_ptr() for t in g), work.data_ptr(), work.numel(), st) == B.OK
        out.append([y, dx, *g])
    assert torch.equal(out[0][0], out[1][0])
    # the weights' sums, and for 96 channels dx's, are cut otherwise: either is within its bound of the exact one
    bounds = L.ffn_backward("silu", *(t.double().cpu().numpy() for t in (x, *w, dy)), "f32")
    for p, q, b in zip(out[0][1:], out[1][1:], bounds):
        assert np.all(np.abs(p.double().cpu().numpy() - q.double().cpu().numpy()) <= 2 * b)
