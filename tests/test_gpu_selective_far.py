"""The selective state space operators where addresses pass 32 bits, on other streams, with scratch made for larger calls, and where calls are long enough to have
every kind of chunk."""
import numpy as np
import pytest
import torch

from oracle import selective as V
from paper_2507_04123_amd import binding as B

import selective_bounds as L
from selective_helpers import DT, TYPES, draw, f64, within, work

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


def _params(c, m, taps):
    return {"w": draw(1, taps, c + 2 * m).cuda(), "bias": draw(2, c + 2 * m).cuda(), "a": -torch.exp(draw(3, c, m)).cuda(), "dt_bias": draw(4, c, shift=-3.0).cuda(),
            "skip": draw(5, c).cuda(), "post": draw(6, c).cuda(), "scale": draw(7, 1).cuda(), "next": draw(8, c).cuda()}


def _all(ctx, dtype, p, rows, x, dy, off, work, backwards, outs):
    """Forward and gradients of all three over rows [x | B | C | dt | gate]; outs: v, s, total, y, ds, drows, dx, dv."""
    c, m = p["a"].shape
    i = c + 2 * m
    v, s, total, y, ds, drows, dx, dv = outs
    k = off.numel() - 1
    f32 = lambda *shape: torch.full(shape, 9.0, device="cuda")  # noqa: E731
    g = {n: torch.full_like(t, 9.0) for n, t in p.items()}
    kept, last, dkept, dh0 = f32(k, len(p["w"]) - 1, i), f32(k, c, m), f32(k, len(p["w"]) - 1, i), f32(k, c, m)
    ctx.causal_conv(dtype, rows[:, :i], p["w"], off, v, bias=p["bias"], backwards=backwards, last=kept)
    cut = lambda t: (t[:, :c], t[:, c:c + m], t[:, c + m:])  # noqa: E731
    xs, b, cc = cut(v)
    dt, z = rows[:, i:i + c], rows[:, i + c:]
    ctx.selective_scan(dtype, xs, dt, p["a"], b, cc, off, s, work, skip=p["skip"], dt_bias=p["dt_bias"], backwards=backwards, last=last)
    ctx.gated_residual(dtype, x, s, p["post"], p["scale"], total, 1e-5, gate=z, next_gain=p["next"], y=y)
    ctx.gated_residual_backward(dtype, x, s, p["post"], p["scale"], 1e-5, None, dx, ds, g["post"], g["scale"], work, gate=z, dgate=drows[:, i + c:],
                                next_gain=p["next"], dy=dy, dnext=g["next"])
    dxs, db, dc = cut(dv)
    ctx.selective_scan_backward(dtype, xs, dt, p["a"], b, cc, off, ds, dxs, drows[:, i:i + c], g["a"], db, dc, work, skip=p["skip"], dskip=g["skip"],
                                dt_bias=p["dt_bias"], ddt_bias=g["dt_bias"], backwards=backwards, dh0=dh0)
    ctx.causal_conv_backward(dtype, rows[:, :i], p["w"], off, dv, drows[:, :i], g["w"], work, bias=p["bias"], dbias=g["bias"], backwards=backwards, dbefore=dkept)
    return [*outs, kept, last, dkept, dh0, *g.values()]


def _outs(n, c, m, td):
    return [torch.full((n, width), -3.0, dtype=td, device="cuda") for width in (c + 2 * m, c, c, c, c, 3 * c + 2 * m, c, c + 2 * m)]


def _scratch(ctx, dtype, n, c, m, taps, fill=0xA5):
    size = max(ctx.selective_scan_work(dtype, n, c, m), ctx.causal_conv_work(dtype, n, c + 2 * m, taps), ctx.gated_residual_work(dtype, n, c))
    return torch.full((size,), fill, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("backwards", [False, True])
def test_rows_beyond_32_bits_of_elements(ctx, backwards):
    """4 200 rows 2^20 + 8 values apart: the last ones lie beyond 2^32 elements."""
    n, c, m, pitch = 4200, 40, 12, (1 << 20) + 8
    p, off = _params(c, m, 4), torch.tensor([0, 1700, n], dtype=torch.int32, device="cuda")
    width = 3 * c + 2 * m
    rows, x, dy = draw(11, n, width, dtype="f16").cuda(), draw(12, n, c, dtype="f16").cuda(), draw(13, n, c, dtype="f16").cuda()
    scratch = _scratch(ctx, B.F16, n, c, m, 4)
    near = _all(ctx, B.F16, p, rows, x, dy, off, scratch, backwards, _outs(n, c, m, torch.float16))
    buffer = torch.empty(n * pitch, dtype=torch.float16, device="cuda")
    wide = buffer.as_strided((n, pitch - 8), (pitch, 1))
    at = 0

    def far(width):
        nonlocal at
        at += width + 3
        return wide[:, at - width - 3:at - 3]

    far_rows, far_x, far_dy = far(width).copy_(rows), far(c).copy_(x), far(c).copy_(dy)
    outs = [far(t.shape[1]) for t in near[:8]]
    got = _all(ctx, B.F16, p, far_rows, far_x, far_dy, off, scratch, backwards, outs)
    assert all(torch.equal(q, r) for q, r in zip(near, got))
    assert torch.equal(far_rows, rows) and torch.equal(far_x, x) and torch.equal(far_dy, dy)


def test_equal_inputs_give_equal_bits_on_other_streams_at_once(ctx):
    n, c, m = 40000, 64, 16
    p, off = _params(c, m, 4), torch.tensor([0, 10, 10, 21000, n], dtype=torch.int32, device="cuda")
    rows, x, dy = draw(11, n, 3 * c + 2 * m, dtype="bf16").cuda(), draw(12, n, c, dtype="bf16").cuda(), draw(13, n, c, dtype="bf16").cuda()
    sets = [(_outs(n, c, m, torch.bfloat16), _scratch(ctx, B.BF16, n, c, m, 4, fill)) for fill in (0, 0xFF, 0x7F)]
    torch.cuda.synchronize()
    results, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for (outs, scratch), stream in zip(sets, [torch.cuda.current_stream()] + streams):
        with torch.cuda.stream(stream):
            results.append(_all(ctx, B.BF16, p, rows, x, dy, off, scratch, False, outs))
    torch.cuda.synchronize()
    for other in results[1:]:
        assert all(torch.equal(q, r) for q, r in zip(results[0], other))


@pytest.mark.parametrize("dtype", TYPES)
def test_scratch_of_the_largest_call_serves_the_smaller_ones(ctx, dtype):
    c, m, td = 33, 9, {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    p, most = _params(c, m, 3), 9000
    scratch = _scratch(ctx, DT[dtype], most, c, m, 3)
    rows, x, dy = draw(1, most, 3 * c + 2 * m, dtype=dtype).cuda(), draw(2, most, c, dtype=dtype).cuda(), draw(3, most, c, dtype=dtype).cuda()
    for n in (most, 8191, 5000, 1025, 1024, 130, 9, 1):
        off = torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda")
        one = _all(ctx, DT[dtype], p, rows[:n], x[:n], dy[:n], off, scratch, False, _outs(n, c, m, td))
        two = _all(ctx, DT[dtype], p, rows[:n], x[:n], dy[:n], off, _scratch(ctx, DT[dtype], n, c, m, 3, 0x11), False, _outs(n, c, m, td))
        assert all(torch.equal(q, r) for q, r in zip(one, two)), n


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("backwards", [False, True])
def test_a_long_call_of_many_spans_against_the_oracle(ctx, dtype, backwards):
    """70 000 rows of few channels: chunks, spans and what enters them all have several, sequences end in all places; states that remember thousands of rows."""
    c, m = 3, 3
    lens = [17000, 0, 5, 1, 130, 2048, 0, 0, 3, 24000, 16, 15, 8, 26774]
    off = np.concatenate([[0], np.cumsum(lens)])
    n, dev = int(off[-1]), torch.from_numpy(off.astype(np.int32)).cuda()
    assert n == 70000
    x, dt, b, cc, dy = (draw(i, n, w, dtype=dtype) for i, w in ((1, c), (2, c), (3, m), (4, m), (5, c)))
    a, bias, skip = -torch.exp(draw(6, c, m, shift=-2.0)), torch.full((c,), -6.0), draw(7, c)
    h0, dlast = draw(8, len(lens), c, m), draw(9, len(lens), c, m)
    g = [t.cuda() for t in (x, dt, a, b, cc)]
    y, last = torch.empty_like(g[0]), torch.empty_like(h0, device="cuda")
    w = work(ctx.selective_scan_work(DT[dtype], n, c, m))
    kw = dict(skip=skip.cuda(), dt_bias=bias.cuda(), backwards=backwards, h0=h0.cuda())
    ctx.selective_scan(DT[dtype], *g, dev, y, w, last=last, **kw)
    e = [f64(t) for t in (x, dt, a, b, cc)]
    args = *e, off, f64(h0), f64(skip), f64(bias)
    ey, el = V.selective_scan(*args, backwards)
    by, bl = L.selective_scan(*args, backwards, dtype)
    within(y, ey, by, "y")
    within(last, el, bl, "last")
    out = {"dx": torch.empty_like(y), "ddt": torch.empty_like(y), "da": torch.empty_like(g[2]), "db": torch.empty_like(g[3]), "dc": torch.empty_like(g[3]),
           "dskip": torch.empty(c, device="cuda"), "ddt_bias": torch.empty(c, device="cuda"), "dh0": torch.empty_like(last)}
    ctx.selective_scan_backward(DT[dtype], *g, dev, dy.cuda(), out["dx"], out["ddt"], out["da"], out["db"], out["dc"], w, dskip=out["dskip"],
                                ddt_bias=out["ddt_bias"], dlast=dlast.cuda(), dh0=out["dh0"], **kw)
    args += f64(dy), f64(dlast), backwards
    exp, bound = V.selective_scan_backward(*args), L.selective_scan_backward(*args, dtype)
    for k in exp:
        within(out[k], exp[k], bound[k], k)
