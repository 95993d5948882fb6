"""What one value of dy that is not finite makes of the feed-forward network's gradients: its own row of dx, its own column of dWd, and the
gates' and up weights' (whose every value has its row's dH as a term)."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from paper_2507_04123_amd import binding as B

import sequence_bounds as L

pytestmark = pytest.mark.gpu

DT = {"f32": (B.F32, torch.float32), "f16": (B.F16, torch.float16), "bf16": (B.BF16, torch.bfloat16)}


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,c,f,row,channel", [(1, 5, 3, 0, 2), (40, 16, 64, 33, 0), (301, 48, 100, 200, 40), (301, 160, 70, 7, 100), (300, 250, 40, 299, 249),
                                                  (20000, 64, 72, 15001, 63), (33000, 100, 40, 17, 31)])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_gradients_of_a_dy_that_is_not_finite(dtype, rows, c, f, row, channel, value):
    dt, td = DT[dtype]
    r = np.random.RandomState(rows + c)
    x, wg, wu, wd, dy = (torch.from_numpy(r.standard_normal(s) * k).to(td) for s, k in
                         (((rows, c), 1), ((c, f), c ** -0.5), ((c, f), c ** -0.5), ((f, c), f ** -0.5), ((rows, c), 1)))
    dirty = dy.clone()
    dirty[row, channel] = value
    ctx = B.Context(1, 1, 1)
    packed = torch.empty(ctx.ffn_packed_size(dt, c, f), dtype=td, device="cuda")
    ctx.ffn_pack(dt, wg.cuda(), wu.cuda(), wd.cuda(), packed)
    work = torch.empty(ctx.ffn_work(dt, rows, c, f), dtype=torch.uint8, device="cuda")

    def run(dy):
        dx, g = torch.empty(rows, c, dtype=td, device="cuda"), [torch.empty(t.shape, dtype=td, device="cuda") for t in (wg, wu, wd)]
        ctx.ffn_backward(dt, B.ACT_SILU, x.cuda(), packed, f, dy.cuda(), dx, *g, work)
        return [t.cpu() for t in (dx, *g)]

    clean, got = run(dy), run(dirty)
    ctx.status_sync()
    ctx.close()
    others, columns = [i for i in range(rows) if i != row], [i for i in range(c) if i != channel]
    assert torch.equal(got[0][others], clean[0][others]) and not torch.isfinite(got[0][row]).any()
    assert not torch.isfinite(got[1]).any() and not torch.isfinite(got[2]).any() and not torch.isfinite(got[3][:, channel]).any()
    args = [t.double().numpy() for t in (x, wg, wu, wd, dy)]
    exp, bound = S.ffn_backward("silu", *args)[3][:, columns], L.ffn_backward("silu", *args, dtype)[3][:, columns]
    bad = ~(np.abs(got[3][:, columns].double().numpy() - exp) <= bound)
    assert not bad.any(), (int(bad.sum()), bad.size)
