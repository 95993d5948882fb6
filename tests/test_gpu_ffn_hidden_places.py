"""Up to 2048 rows the hidden values of 16-bit networks and their gradients are held in two parts, to the square of the type's unit roundoff: the
results are as near as fp32 hidden values make them, and one rounding to the result's own type."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from paper_2507_04123_amd import binding as B

import sequence_bounds as L

pytestmark = pytest.mark.gpu

DT = {"f16": (B.F16, torch.float16), "bf16": (B.BF16, torch.bfloat16)}


def _two_parts(v, dtype):
    """How far a value held in two parts may be off: the first leaves u |v| over at most, the second u of that (or half a unit of the smallest number)."""
    return L.U[dtype] ** 2 * np.abs(v) + L.TINY[dtype]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,c,f", [(1, 8, 16), (5, 32, 30), (10, 16, 64), (24, 128, 512), (70, 13, 16), (33, 200, 40), (40, 256, 300), (300, 96, 100), (515, 160, 90),
                                      (2048, 64, 72)])
def test_hidden_values_in_two_parts(dtype, act, rows, c, f):
    dt, td = DT[dtype]
    r = np.random.RandomState(rows + c)
    x, wg, wu, wd, dy = (torch.from_numpy(r.standard_normal(s) * k).to(td) for s, k in
                         (((rows, c), 1), ((c, f), c ** -0.5), ((c, f), c ** -0.5), ((f, c), f ** -0.5), ((rows, c), 1)))
    ctx, code = B.Context(1, 1, 1), B.ACT_SILU if act == "silu" else B.ACT_GELU
    packed = torch.full((ctx.ffn_packed_size(dt, c, f),), float("nan"), dtype=td, device="cuda")
    ctx.ffn_pack(dt, wg.cuda(), wu.cuda(), wd.cuda(), packed)
    y, dx, *g = (torch.full(t.shape, 7.0, dtype=td, device="cuda") for t in (x, x, wg, wu, wd))
    work = torch.empty(ctx.ffn_work(dt, rows, c, f), dtype=torch.uint8, device="cuda")
    ctx.ffn(dt, code, x.cuda(), packed, f, y)
    ctx.ffn_backward(dt, code, x.cuda(), packed, f, dy.cuda(), dx, *g, work)
    ctx.status_sync()
    ctx.close()
    a = xs, wgs, wus, wds, dys = [t.double().numpy() for t in (x, wg, wu, wd, dy)]
    value, slope = S.activate(act, xs @ wgs)
    up, dh = xs @ wus, dys @ wds.T
    eh, edg, edu = (_two_parts(v, dtype) for v in (value * up, dh * up * slope, dh * value))
    xa, dya = np.abs(xs), np.abs(dys)
    more = (eh @ np.abs(wds), edg @ np.abs(wgs.T) + edu @ np.abs(wus.T), xa.T @ edg, xa.T @ edu, eh.T @ dya)
    exp = (S.ffn(act, *a[:4]), *S.ffn_backward(act, *a))
    inner = (L.ffn(act, *a[:4], np.zeros_like(xs), "f32"), *L.ffn_backward(act, *a, "f32"))
    for got, e, b, m, what in zip((y, dx, *g), exp, inner, more, ("y", "dx", "dwg", "dwu", "dwd")):
        got = got.double().cpu().numpy()
        bad = ~(np.abs(got - e) <= L.rounded(e, b + m, dtype))
        assert not bad.any(), (what, int(bad.sum()), bad.size, got[bad][:3], e[bad][:3])
