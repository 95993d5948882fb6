"""The gated residual with its norms, and its gradients, against the oracle in 64 bits within the bounds of the number formats; its refusals."""
import pytest
import torch

from oracle import selective as V
from paper_2507_04123_amd import binding as B

import selective_bounds as L
from selective_helpers import DT, TYPES, draw, f64, like, rows, within, work

pytestmark = pytest.mark.gpu
WIDTHS = [1, 3, 8, 16, 47, 64, 90, 128, 160, 250, 384, 511, 512, 1000, 1024]


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


def _case(seed, n, c, dtype, gate=True):
    p = {"x": draw(seed, n, c, dtype=dtype), "branch": draw(seed + 1, n, c, scale=2.0, shift=0.5, dtype=dtype),
         "gate": draw(seed + 2, n, c, scale=2.0, dtype=dtype) if gate else None, "post": draw(seed + 3, c, scale=0.3, shift=1.0),
         "scale": draw(seed + 4, 1, scale=0.3, shift=0.6), "next": draw(seed + 5, c, scale=0.3, shift=1.0)}
    p["branch"][n // 2] = 0
    return p


def _oracle(p):
    return [f64(p[k]) if p[k] is not None else None for k in ("x", "branch", "gate", "post", "scale", "next")] + [1e-5]


def _forward(ctx, p, dtype, how, with_y=True):
    g = {k: (rows(t, how) if t.dim() == 2 else t.cuda()) if t is not None else None for k, t in p.items()}
    total, y = like(p["x"], how), like(p["x"], how) if with_y else None
    ctx.gated_residual(DT[dtype], g["x"], g["branch"], g["post"], g["scale"], total, 1e-5, gate=g["gate"], next_gain=g["next"] if with_y else None, y=y)
    return g, total, y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", WIDTHS)
def test_forward(ctx, dtype, c):
    for n, how, gate, with_y in ((1, "packed", True, True), (37, "slice", False, True), (301, "odd", True, True), (64, "packed", True, False)):
        p = _case(c, n, c, dtype, gate)
        _, total, y = _forward(ctx, p, dtype, how, with_y)
        args = _oracle(p)
        et, ey = V.gated_residual(*args)
        bt, by = L.gated_residual(*args, dtype)
        within(total, et, bt, "sum")
        if with_y:
            within(y, ey, by, "y")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", WIDTHS)
def test_backward(ctx, dtype, c):
    for n, how, gate, with_sum, with_y in ((1, "packed", True, True, True), (37, "slice", False, True, True), (700, "odd", True, True, True),
                                           (1200, "packed", True, False, True), (65, "packed", True, True, False)):
        p = _case(c + 7, n, c, dtype, gate)
        dsum, dy = draw(c, n, c, dtype=dtype), draw(c + 1, n, c, dtype=dtype)
        g = {k: (rows(t, how) if t.dim() == 2 else t.cuda()) if t is not None else None for k, t in p.items()}
        out = {k: like(p["x"], how) for k in ("dx", "dbranch", "dgate")}
        vec = {k: torch.full((size,), 9.0, device="cuda") for k, size in (("dpost", c), ("dscale", 1), ("dnext", c))}
        ctx.gated_residual_backward(DT[dtype], g["x"], g["branch"], g["post"], g["scale"], 1e-5, rows(dsum, how) if with_sum else None, out["dx"],
                                    out["dbranch"], vec["dpost"], vec["dscale"], work(ctx.gated_residual_work(DT[dtype], n, c)), gate=g["gate"],
                                    dgate=out["dgate"] if gate else None, next_gain=g["next"] if with_y else None,
                                    dy=rows(dy, how) if with_y else None, dnext=vec["dnext"] if with_y else None)
        args = _oracle(p) + [f64(dsum) * with_sum, f64(dy) * with_y]
        exp, bound = V.gated_residual_backward(*args), L.gated_residual_backward(*args, dtype)
        for k in exp:
            if (k != "dgate" or gate) and (k != "dnext" or with_y):
                within({**out, **vec}[k], exp[k], bound[k], k)
            elif k == "dgate":
                assert (out[k] == -3).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_device_count_in_place_and_no_rows(ctx, dtype):
    n, c = 50, 64
    p = _case(3, n, c, dtype)
    g, whole_total, whole_y = _forward(ctx, p, dtype, "packed")
    dsum, dy = draw(5, n, c, dtype=dtype).cuda(), draw(6, n, c, dtype=dtype).cuda()
    for count in (0, 1, 33, 50, 99, -4):
        k, dn = min(max(count, 0), n), torch.tensor([count], dtype=torch.int32, device="cuda")
        x, b = g["x"].clone(), g["branch"].clone()
        x[k:], b[k:] = float("nan"), float("nan")                        # rows beyond the count are not looked at
        keep_x, keep_b = x.clone(), b.clone()
        ctx.gated_residual(DT[dtype], x, b, g["post"], g["scale"], x, 1e-5, gate=g["gate"], next_gain=g["next"], y=b, n=dn)
        assert torch.equal(x[:k], whole_total[:k]) and torch.equal(b[:k], whole_y[:k])
        assert torch.isnan(x[k:]).all() and torch.isnan(b[k:]).all()
        results = []
        for place in (False, True):
            x, b, z, s, d = keep_x.clone(), keep_b.clone(), g["gate"].clone(), dsum.clone(), dy.clone()
            outs = (s, b, z) if place else tuple(torch.zeros_like(x) for _ in range(3))
            vec = [torch.full((size,), 9.0, device="cuda") for size in (c, 1, c)]
            ctx.gated_residual_backward(DT[dtype], x, b, g["post"], g["scale"], 1e-5, s, outs[0], outs[1], vec[0], vec[1],
                                        work(ctx.gated_residual_work(DT[dtype], n, c)), gate=z, dgate=outs[2], next_gain=g["next"], dy=d, dnext=vec[2],
                                        n=dn)
            results.append([t[:k] for t in outs] + vec)
            assert all(torch.isfinite(t).all() for t in results[-1])
        assert all(torch.equal(a, b) for a, b in zip(*results))
        if k == 0:
            assert not any(t.any() for t in results[0])


def test_refusals(ctx):
    n, c = 8, 16
    p = _case(1, n, c, "f16")
    g, total, y = _forward(ctx, p, "f16", "packed")
    f = lambda x=g["x"], b=g["branch"], t=total, **k: ctx.gated_residual(B.F16, x, b, g["post"], g["scale"], t, k.pop("eps", 1e-5), **k)  # noqa: E731
    for bad in ({"eps": -1.0}, {"eps": float("nan")}, {"y": y}, {"next_gain": g["next"]}, {"y": total, "next_gain": g["next"]}):
        with pytest.raises(B.Emc2Error):
            f(**bad)
    wide = torch.zeros((n, 24), dtype=torch.float16, device="cuda")
    with pytest.raises(B.Emc2Error, match="overlap"):
        f(x=wide[:, :16], t=wide[:, 8:])
    for bad in ({"x": g["x"].float()}, {"gate": g["gate"][:, :8]}, {"gate": g["gate"][:4]}):
        with pytest.raises(ValueError):
            f(**bad)
    big = torch.zeros((1, 1025), dtype=torch.float16, device="cuda")
    ones = torch.ones(1025, device="cuda")
    with pytest.raises(B.Emc2Error) as e:
        ctx.gated_residual(B.F16, big, big, ones, g["scale"], torch.zeros_like(big), 1e-5)
    assert e.value.status == B.ERR_UNSUPPORTED and ctx.gated_residual_work(B.F16, 4, 1025) == -1
    grads = [torch.zeros_like(g["x"]) for _ in range(3)]
    w = work(ctx.gated_residual_work(B.F16, n, c))
    back = lambda dt=total, **k: ctx.gated_residual_backward(  # noqa: E731
        B.F16, g["x"], g["branch"], g["post"], g["scale"], 1e-5, dt, grads[0], grads[1], torch.zeros(c, device="cuda"), torch.zeros(1, device="cuda"),
        k.pop("work", w), **k)
    back()
    for bad in ({"dt": None}, {"gate": g["gate"]}, {"dgate": grads[2]}, {"dy": y}, {"dy": y, "next_gain": g["next"]},
                {"gate": g["gate"], "dgate": grads[0]}):
        with pytest.raises(B.Emc2Error):
            back(**bad)
    with pytest.raises(ValueError):
        back(work=w[:-4])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [2, 4, 5, 7, 9, 11, 12, 13, 15, 18, 20, 24, 27, 31, 32, 33])
def test_narrow_rows(ctx, dtype, c):
    """Rows that two and four lanes hold, in whole vectors and with a last one moved back."""
    test_forward(ctx, dtype, c)
    test_backward(ctx, dtype, c)


@pytest.mark.parametrize("dtype", TYPES)
def test_more_narrow_rows_than_all_blocks_hold_at_once(ctx, dtype):
    n, c = 140001, 12
    p = _case(3, n, c, dtype)
    dsum, dy = draw(4, n, c, dtype=dtype), draw(5, n, c, dtype=dtype)
    g, total, y = _forward(ctx, p, dtype, "packed")
    args = _oracle(p)
    for got, exp, bound in zip((total, y), V.gated_residual(*args), L.gated_residual(*args, dtype)):
        within(got, exp, bound, "forward")
    out = {k: like(p["x"], "packed") for k in ("dx", "dbranch", "dgate")}
    out.update({k: torch.full((size,), 9.0, device="cuda") for k, size in (("dpost", c), ("dscale", 1), ("dnext", c))})
    ctx.gated_residual_backward(DT[dtype], g["x"], g["branch"], g["post"], g["scale"], 1e-5, dsum.cuda(), out["dx"], out["dbranch"], out["dpost"], out["dscale"],
                                work(ctx.gated_residual_work(DT[dtype], n, c)), gate=g["gate"], dgate=out["dgate"], next_gain=g["next"], dy=dy.cuda(),
                                dnext=out["dnext"])
    args += [f64(dsum), f64(dy)]
    exp, bound = V.gated_residual_backward(*args), L.gated_residual_backward(*args, dtype)
    for k in exp:
        within(out[k], exp[k], bound[k], k)
