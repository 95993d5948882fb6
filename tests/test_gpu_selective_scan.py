"""The selective state space scan, its gradients and its form for one row per sequence, against the oracle in 64 bits within the bounds of the number formats;
its refusals."""
import numpy as np
import pytest
import torch

from oracle import selective as V
from paper_2507_04123_amd import binding as B

import selective_bounds as L
from selective_helpers import DT, LENGTHS, TYPES, draw, f64, like, offsets, rows, within, work

pytestmark = pytest.mark.gpu
GRADS = ("dx", "ddt", "da", "db", "dc", "dskip", "ddt_bias", "dh0")


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


def _case(seed, lens, c, m, dtype, extras=True):
    """Steps of many sizes, a few that forget everything; states that remember one to some hundred rows."""
    off, dev = offsets(lens)
    n, s = int(off[-1]), len(lens)
    p = {"x": draw(seed, n, c, dtype=dtype), "dt": draw(seed + 1, n, c, scale=1.5, dtype=dtype), "b": draw(seed + 3, n, m, dtype=dtype),
         "c": draw(seed + 4, n, m, dtype=dtype), "dy": draw(seed + 5, n, c, dtype=dtype), "dlast": draw(seed + 6, s, c, m)}
    p["dt"][7::23] *= 8
    p["a"] = -torch.exp(draw(seed + 2, c, m, scale=1.2)).float()
    p["skip"], p["dt_bias"], p["h0"] = (draw(seed + 7, c), draw(seed + 8, c, shift=-3.0), draw(seed + 9, s, c, m)) if extras else (None, None, None)
    e = {k: f64(t) if t is not None else None for k, t in p.items()}
    if not extras:
        e["skip"], e["dt_bias"], e["h0"], e["dlast"] = np.zeros(c), np.zeros(c), np.zeros((s, c, m)), np.zeros((s, c, m))
    return off, dev, p, e


def _gpu(p, how):
    return {k: (rows(t, how) if k in ("x", "dt", "b", "c", "dy") else t.cuda()) if t is not None else None for k, t in p.items()}


def _forward(ctx, dtype, g, p, dev, how, backwards):
    n, c = p["x"].shape
    y, last = like(p["x"], how), torch.full(p["dlast"].shape, -5.0, device="cuda")
    w = work(ctx.selective_scan_work(DT[dtype], n, c, p["a"].shape[1]))
    ctx.selective_scan(DT[dtype], g["x"], g["dt"], g["a"], g["b"], g["c"], dev, y, w, skip=g["skip"], dt_bias=g["dt_bias"], backwards=backwards, h0=g["h0"],
                       last=last)
    return y, last


def _backward(ctx, dtype, g, p, dev, how, backwards, extras=True):
    n, c = p["x"].shape
    m = p["a"].shape[1]
    out = {"dx": like(p["x"], how), "ddt": like(p["x"], how), "db": like(p["b"], how), "dc": like(p["b"], how), "da": torch.full((c, m), 9.0, device="cuda")}
    if extras:
        out.update({k: torch.full((c,), 9.0, device="cuda") for k in ("dskip", "ddt_bias")}, dh0=torch.full(p["dlast"].shape, 9.0, device="cuda"))
    w = work(ctx.selective_scan_work(DT[dtype], n, c, m))
    ctx.selective_scan_backward(DT[dtype], g["x"], g["dt"], g["a"], g["b"], g["c"], dev, g["dy"], out["dx"], out["ddt"], out["da"], out["db"], out["dc"], w,
                                skip=g["skip"], dskip=out.get("dskip"), dt_bias=g["dt_bias"], ddt_bias=out.get("ddt_bias"), backwards=backwards, h0=g["h0"],
                                dlast=g["dlast"] if extras else None, dh0=out.get("dh0"))
    return out


def _check(ctx, dtype, lens, c, m, how="packed", backwards=False, extras=True):
    off, dev, p, e = _case(c + m, lens, c, m, dtype, extras)
    g = _gpu(p, how)
    y, last = _forward(ctx, dtype, g, p, dev, how, backwards)
    args = [e[k] for k in ("x", "dt", "a", "b", "c")] + [off] + [e[k] for k in ("h0", "skip", "dt_bias")]
    ey, el = V.selective_scan(*args, backwards)
    by, bl = L.selective_scan(*args, backwards, dtype)
    within(y, ey, by, "y")
    within(last, el, bl, "last")
    out = _backward(ctx, dtype, g, p, dev, how, backwards, extras)
    args += [e["dy"], e["dlast"], backwards]
    exp, bound = V.selective_scan_backward(*args), L.selective_scan_backward(*args, dtype)
    for k in out:
        within(out[k], exp[k], bound[k], k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", LENGTHS)
def test_lengths(ctx, dtype, name):
    _check(ctx, dtype, LENGTHS[name], 10, 8)
    _check(ctx, dtype, LENGTHS[name], 5, 16, "odd", True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 7, 8, 12, 15, 16, 17, 24, 31, 32, 33, 48, 63, 64])
def test_states(ctx, dtype, m):
    _check(ctx, dtype, [33, 0, 70, 2], 9, m, "slice", m % 2 == 0)
    _check(ctx, dtype, [1100, 3, 40], 6, m, "packed", m % 3 == 0, extras=m % 4 != 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [1, 2, 31, 32, 33, 63, 64, 65, 90, 130, 257, 320])
def test_widths(ctx, dtype, c):
    _check(ctx, dtype, [33, 0, 50, 2], c, 4, "odd" if c % 2 else "slice", c % 3 == 0)
    _check(ctx, dtype, [40, 3], c, 16, "packed", extras=c % 2 == 0)
    if c < 140:
        _check(ctx, dtype, [600, 0, 500], c, 6)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [520, 1100])
def test_channels_of_several_blocks(ctx, dtype, c):
    _check(ctx, dtype, [20, 0, 9], c, 16)
    _check(ctx, dtype, [9, 12], c, 40, "odd", True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c,m", [(1, 1), (16, 16), (37, 7), (64, 16), (33, 64), (128, 30)])
def test_step_moves_on_where_a_run_ended(ctx, dtype, c, m):
    streams, first, more = 5, 6, 4
    off, dev, p, e = _case(2, [first + more] * streams, c, m, dtype)
    pick = lambda t, lo, hi: t.reshape(streams, first + more, -1)[:, lo:hi].reshape(streams * (hi - lo), -1).contiguous()  # noqa: E731
    head = {k: pick(t, 0, first) if k in ("x", "dt", "b", "c", "dy") else t for k, t in p.items()}
    g = _gpu(head, "packed")
    _, state = _forward(ctx, dtype, g, head, offsets([first] * streams)[1], "packed", False)
    for t in range(first, first + more):
        now = {k: pick(p[k], t, t + 1) for k in ("x", "dt", "b", "c")}
        r = {k: rows(v, "odd") for k, v in now.items()}
        y, to = torch.empty((streams, c), dtype=now["x"].dtype, device="cuda"), state if t % 2 else torch.empty_like(state)
        past = f64(state)
        ctx.selective_scan_step(DT[dtype], r["x"], r["dt"], g["a"], r["b"], r["c"], state, to, y, skip=g["skip"], dt_bias=g["dt_bias"])
        args = [f64(now["x"]), f64(now["dt"]), e["a"], f64(now["b"]), f64(now["c"]), np.arange(streams + 1), past, e["skip"], e["dt_bias"]]
        ey, el = V.selective_scan(*args)
        by, bl = L.selective_scan(*args, False, dtype)
        within(y, ey, by, "y")
        within(to, el, bl, "h")
        state = to


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_are_those_of_the_outputs_themselves(ctx, dtype):
    """fp32 and 16-bit gradients along random directions against central differences of the definition in 64 bits: within the gradients' own bounds along the direction."""
    lens, c, m = [30, 0, 45, 1], 7, 5
    off, dev, p, e = _case(3, lens, c, m, dtype)
    out = _backward(ctx, dtype, _gpu(p, "packed"), p, dev, "packed", False)
    names = {"dx": "x", "ddt": "dt", "da": "a", "db": "b", "dc": "c", "dskip": "skip", "ddt_bias": "dt_bias", "dh0": "h0"}
    order = ("x", "dt", "a", "b", "c")
    args = [e[k] for k in order] + [off] + [e[k] for k in ("h0", "skip", "dt_bias")] + [e["dy"], e["dlast"], False]
    bound = L.selective_scan_backward(*args, dtype)

    def loss(q):
        y, last = V.selective_scan(*[q[k] for k in order], off, q["h0"], q["skip"], q["dt_bias"])
        return (y * e["dy"]).sum() + (last * e["dlast"]).sum()

    for i, (k, name) in enumerate(names.items()):
        d = np.random.RandomState(i).standard_normal(e[name].shape)
        num = (loss({**e, name: e[name] + 1e-5 * d}) - loss({**e, name: e[name] - 1e-5 * d})) / 2e-5
        assert abs(num - (f64(out[k]) * d).sum()) <= (bound[k] * np.abs(d)).sum() + 1e-7 * (1 + np.abs(f64(out[k]) * d).sum()), k


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [[40, 30, 0, 20], [700, 600, 0, 900]])
def test_nonfinite_values_stay_in_their_sequence_and_channel(ctx, dtype, lens):
    c, m = 9, 12
    off, dev, p, e = _case(5, lens, c, m, dtype)
    out = []
    for poison in (False, True):
        if poison:
            p["x"][10, 2] = float("inf")                                 # from row 10 of the first sequence on, channel 2
            p["dt"][off[1] + 5, 4] = float("nan")                        # from there to the second sequence's end, channel 4
            p["dy"][off[1] + 9, 6] = float("nan")                        # before there, channel 6's gradients
        g = _gpu(p, "packed")
        out.append((*_forward(ctx, dtype, g, p, dev, "packed", False), _backward(ctx, dtype, g, p, dev, "packed", False)))
    (y0, l0, g0), (y1, l1, g1) = out
    hit = torch.zeros_like(y0, dtype=torch.bool)
    hit[10:off[1], 2] = True
    hit[off[1] + 5:off[2], 4] = True
    assert torch.equal(y0[~hit], y1[~hit]) and not torch.isfinite(y1[10, 2]) and not torch.isfinite(y1[off[1] + 5:off[2], 4]).any()
    states = torch.ones_like(l0, dtype=torch.bool)
    states[0, 2] = states[1, 4] = False
    assert torch.equal(l0[states], l1[states])
    for k in ("dx", "ddt"):                                              # rows and channels that none of the three reach
        far = torch.ones_like(y0, dtype=torch.bool)
        far[:off[1], 2] = False
        far[off[1]:off[2], 4] = False
        far[off[1]:off[1] + 10, 6] = False
        assert torch.equal(g0[k][far], g1[k][far]), k
    assert torch.equal(g0["db"][off[2]:], g1["db"][off[2]:]) and torch.equal(g0["dc"][off[2]:], g1["dc"][off[2]:])
    other = [i for i in range(c) if i not in (2, 4, 6)]
    for k in ("da", "dskip", "ddt_bias"):
        assert torch.equal(g0[k][other], g1[k][other]), k


def test_an_infinite_row_gives_what_the_formula_gives(ctx):
    """Padded states take no part: with all B of one sign and C of one sign an infinite row makes y infinite, not NaN."""
    for m in (3, 13, 20):
        for n in (50, 1500):
            off, dev = offsets([n])
            x, dt, b = torch.ones((n, 5)), torch.zeros((n, 5)), torch.ones((n, m))
            x[7, 3] = float("inf")
            a = -torch.ones((5, m)) * 1e-3
            y = torch.empty((n, 5), device="cuda")
            ctx.selective_scan(B.F32, x.cuda(), dt.cuda(), a.cuda(), b.cuda(), b.cuda(), dev, y, work(ctx.selective_scan_work(B.F32, n, 5, m)))
            assert torch.isinf(y[7:, 3]).all() and torch.isfinite(y[:7]).all() and torch.isfinite(y[:, [0, 1, 2, 4]]).all()


def test_in_place_and_slices_of_one_buffer(ctx):
    c, m = 24, 8
    for lens in ([30, 11], [900, 800]):
        off, dev, p, _ = _case(4, lens, c, m, "f16")
        n = int(off[-1])
        g = _gpu(p, "packed")
        y, last = _forward(ctx, "f16", g, p, dev, "packed", True)
        d = _backward(ctx, "f16", g, p, dev, "packed", True)
        wide = torch.cat([g["x"], g["b"], g["c"], g["dt"]], 1)
        x, b, cc, dt = wide[:, :c], wide[:, c:c + m], wide[:, c + m:c + 2 * m], wide[:, c + 2 * m:]
        w = work(ctx.selective_scan_work(B.F16, n, c, m))
        dx, ddt, db = g["dy"].clone(), dt, torch.empty_like(g["b"])
        grads = torch.empty((n, 2 * m), dtype=torch.float16, device="cuda")
        da = torch.empty_like(g["a"])
        kw = dict(skip=g["skip"], dt_bias=g["dt_bias"], backwards=True, h0=g["h0"])
        ctx.selective_scan_backward(B.F16, x, dt, g["a"], b, cc, dev, dx, dx, dt, da, grads[:, :m], grads[:, m:], w, dlast=g["dlast"], **kw)
        assert torch.equal(dx, d["dx"]) and torch.equal(dt, d["ddt"]) and torch.equal(grads[:, :m], d["db"]) and torch.equal(grads[:, m:], d["dc"])
        assert torch.equal(da, d["da"])
        dt.copy_(g["dt"])
        ctx.selective_scan(B.F16, x, dt, g["a"], b, cc, dev, x, w, **kw)
        assert torch.equal(x, y)


def test_rows_beyond_the_last_sequence_and_too_many(ctx):
    c, m = 12, 8
    for n, cap in ((25, 40), (1300, 1500)):
        off, dev, p, _ = _case(6, [n // 2, n - n // 2], c, m, "f16")
        more = {k: torch.cat([t, torch.full((cap - n, t.shape[1]), float("nan"), dtype=t.dtype)]) if k in ("x", "dt", "b", "c", "dy") else t for k, t in p.items()}
        g, gm = _gpu(p, "packed"), _gpu(more, "packed")
        y, last = _forward(ctx, "f16", g, p, dev, "packed", False)
        ym, lastm = _forward(ctx, "f16", gm, more, dev, "packed", False)
        assert torch.allclose(y.float(), ym[:n].float(), rtol=2e-3, atol=2e-3) and (ym[n:] == -3).all() and torch.isfinite(lastm).all()
        d = _backward(ctx, "f16", gm, more, dev, "packed", False)
        assert all((d[k][n:] == -3).all() and torch.isfinite(d[k][:n]).all() for k in ("dx", "ddt", "db", "dc"))
        assert all(torch.isfinite(d[k]).all() for k in ("da", "dskip", "ddt_bias", "dh0"))
        ctx.status_sync()
        # offsets that do not rise, or pass the rows, stay within them
        for bad in ([5, cap // 2, 10, cap], [0, -7, 2 * cap, 33], [cap, 0, cap, 0], [cap - 1, cap - 2, cap - 3, cap - 4], [0, 1, 2, cap + 1]):
            off = torch.tensor(bad, dtype=torch.int32, device="cuda")
            three = {**gm, **{k: torch.ones((3, c, m), device="cuda") for k in ("h0", "dlast")}}
            q = {**more, "dlast": torch.zeros(3, c, m)}
            for back in (False, True):
                _forward(ctx, "f16", three, q, off, "packed", back)
                _backward(ctx, "f16", three, q, off, "packed", back)
        with pytest.raises(B.Emc2Error) as e:
            ctx.status_sync()
        assert e.value.status == B.ERR_CAPACITY
        assert torch.equal(_forward(ctx, "f16", g, p, dev, "packed", False)[0], y)


def test_refusals(ctx):
    c, m, n = 16, 8, 10
    off, dev, p, _ = _case(1, [n], c, m, "f16")
    g = _gpu(p, "packed")
    y, w = torch.empty_like(g["x"]), work(ctx.selective_scan_work(B.F16, n, c, m))
    run = lambda **k: ctx.selective_scan(B.F16, *[k.get(q, g[q]) for q in ("x", "dt", "a", "b", "c")], dev, k.get("y", y), k.get("w", w),  # noqa: E731
                                         h0=g["h0"], last=k.get("last"))
    run()
    square = torch.zeros((n, c), dtype=torch.float16, device="cuda")
    wide = torch.zeros((n, 40), dtype=torch.float16, device="cuda")
    a65 = torch.zeros((c, 65), device="cuda")
    b65 = torch.zeros((n, 65), dtype=torch.float16, device="cuda")
    for bad in ({"last": g["h0"]}, {"b": wide[:, :m], "y": wide[:, 4:4 + c]}, {"x": wide[:, :c], "y": wide[:, 8:8 + c]}, {"a": a65, "b": b65, "c": b65}):
        with pytest.raises((B.Emc2Error, ValueError)):
            run(**bad)
    for bad in ({"b": g["b"].float()}, {"b": g["b"][:5]}, {"c": square}, {"a": g["a"].half()}, {"dt": g["dt"][:, :8]}, {"w": w[:8]}):
        with pytest.raises(ValueError):
            run(**bad)
    out = {k: torch.empty_like(g[q]) for k, q in (("dx", "x"), ("ddt", "dt"), ("db", "b"), ("dc", "c"), ("da", "a"))}
    back = lambda **k: ctx.selective_scan_backward(B.F16, *[g[q] for q in ("x", "dt", "a", "b", "c")], dev, g["dy"], *[k.get(q, out[q]) for q in (  # noqa: E731
        "dx", "ddt", "da", "db", "dc")], w, dskip=k.get("dskip"), h0=g["h0"], dlast=g["dlast"], dh0=k.get("dh0"))
    back()
    for bad in ({"dx": out["ddt"]}, {"db": g["b"]}, {"dc": out["db"]}, {"dh0": g["h0"]}, {"dh0": g["dlast"]}, {"dskip": torch.zeros(c, device="cuda")}):
        with pytest.raises(B.Emc2Error):
            back(**bad)
    h = torch.zeros((n, c, m), device="cuda")
    both = torch.zeros(2 * n * c * m, device="cuda")
    with pytest.raises(B.Emc2Error):
        ctx.selective_scan_step(B.F16, g["x"], g["dt"], g["a"], g["b"], g["c"], both[:n * c * m].view(n, c, m), both[4:4 + n * c * m].view(n, c, m), y)
    with pytest.raises(ValueError):
        ctx.selective_scan_step(B.F16, g["x"], g["dt"], g["a"], g["b"], g["c"], h[:5], h, y)
    one = {q: g[q][:1] for q in ("x", "dt", "b", "c")}
    far = torch.as_strided(torch.zeros(c, dtype=torch.float16, device="cuda"), (1, c), ((1 << 26) + 1, 1))
    with pytest.raises(B.Emc2Error, match="2\\^26"):
        ctx.selective_scan(B.F16, far, one["dt"], g["a"], one["b"], one["c"], dev, y[:1], w)
    assert ctx.selective_scan_work(B.F16, n, c, 65) == -1 and ctx.selective_scan_work(B.I8, n, c, m) == -1
