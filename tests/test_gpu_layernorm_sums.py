"""The layer norm's weight gradients are sums over all rows.  fp32 sums lose at most a unit roundoff for every addition behind a term, so
the depth of the tree that they are added in is what can be held to."""
import numpy as np
import pytest
import torch

from paper_2507_04123_amd import binding as B

pytestmark = pytest.mark.gpu

TD = {B.F32: torch.float32, B.F16: torch.float16, B.BF16: torch.bfloat16}


@pytest.mark.parametrize("dtype,rows,c", [(B.F32, 20011, 90), (B.F32, 40000, 33), (B.F16, 40000, 100), (B.F16, 80000, 64), (B.BF16, 40000, 128),
                                          (B.BF16, 10000, 512)])
@pytest.mark.parametrize("first", [0, 777])
def test_weight_sums_in_few_additions(dtype, rows, c, first):
    """One row of dy is 1 (times a power of two), every other one so small that what a block has of them just fails to change it.  Every sum
    below a block's is exact; added one after the other, the blocks' leave the large value as it is.  At these sizes a lane has two rows (one
    addition), then there are up to 3 over the lanes, 3 over the waves, 3 + 5 over the blocks that a thread adds and 5 over the threads: 20, of half a
    unit in the last place of a sum that is at most the sum of magnitudes."""
    td = TD[dtype]
    small = 2.0 ** -(24 + int(np.ceil(np.log2(rows / 1250))))                          # 1250 blocks
    dy = torch.full((rows, c), small * 2.0 ** 14, dtype=td)
    dy[first] = 2.0 ** 14
    x = torch.tensor([1.0, -1.0] * ((c + 1) // 2))[:c].to(td).repeat(rows, 1)
    x[:, c - 1] = 0 if c % 2 else x[:, c - 1]                                         # mean 0, every row the same
    ctx = B.Context(1, 1, 1)
    dx, dg, db = torch.empty(rows, c, dtype=td, device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    work = torch.empty(ctx.layernorm_work(dtype, rows, c), dtype=torch.uint8, device="cuda")
    ctx.layernorm_backward(dtype, x.cuda(), torch.ones(c, device="cuda"), 0.0, dy.cuda(), dx, dg, db, work)
    ctx.status_sync()
    ctx.close()
    d = dy.double().sum(0).numpy()
    u = 2.0 ** -24
    assert np.all(np.abs(db.double().cpu().numpy() - d) <= 20 * u * d)
    # dgamma's terms are dy xh: xh itself is computed, the same for every row, to a few roundings (a mean of 0, the squares' sum, its root, a product)
    xh = x[0].double().numpy() / np.sqrt((x[0].double().numpy() ** 2).mean())
    assert np.all(np.abs(dg.double().cpu().numpy() - d * xh) <= (20 + 2 + 16) * u * d * np.abs(xh))
