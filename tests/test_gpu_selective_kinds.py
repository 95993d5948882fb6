"""An infinity or NaN in one value of one operand of the selective operators: every value of every result is infinite, NaN or finite where the formula in 64 bits makes it so."""
import numpy as np
import pytest
import torch

from oracle import selective as V
from paper_2507_04123_amd import binding as B

from selective_helpers import DT, draw, f64, offsets, work
from selective_infinite import case, oracle, run

pytestmark = pytest.mark.gpu
TYPES = ["f32", "f16"]
VALUES = [float("inf"), -float("inf"), float("nan")]


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


def _kind(v):
    return np.where(np.isnan(v), 2, np.where(np.isinf(v), np.sign(v), 0))


def _check(got, exp, what):
    got = f64(got)
    free = np.isfinite(exp) & (np.abs(exp) > 60000.0)                    # f16 ends there
    same = (_kind(got) == _kind(exp)) | free
    assert same.all(), (what, int((~same).sum()), tuple(np.argwhere(~same)[0]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("what", ["x", "dt", "b", "c", "dy", "h0", "dlast", "a"])
def test_scan(ctx, dtype, what):
    for c, m, lens in ((1, 3, [40, 30, 0, 20]), (9, 13, [400, 600, 0, 60]), (40, 16, [40, 30, 0, 20]), (33, 20, [40, 300, 0, 20]), (17, 40, [400, 30, 0, 20])):
        off, dev = offsets(lens)
        for value in VALUES if what != "a" else [0.0]:                   # (a of 0: states that forget nothing, whatever the step)
            for at, backwards in ((11, False), (16, True)):
                p, row = case(lens, c, m, dtype), int(off[1]) + at
                if what == "a":
                    p["a"][0, 0], p["dt"][row, 0] = value, float("inf")
                elif what in ("h0", "dlast"):
                    p[what][1, 0, m // 2] = value
                else:
                    p[what][row, 0] = value
                y, last, out = run(ctx, dtype, p, dev, backwards)
                args, grads = oracle(p, off, backwards)
                with np.errstate(all="ignore"):
                    ey, el = V.selective_scan(*args, backwards)
                    exp = V.selective_scan_backward(*grads)
                tag = c, m, value, backwards
                _check(y, ey, ("y", *tag))
                _check(last, el, ("last", *tag))
                for k in exp:
                    _check(out[k], exp[k], (k, *tag))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("what", ["x", "w", "bias", "before", "dy", "dlast"])
def test_conv(ctx, dtype, what):
    for c, taps, lens in ((1, 4, [9, 12, 0, 20, 1]), (9, 3, [300, 0, 400]), (24, 8, [9, 12, 0, 20, 1]), (100, 4, [300, 0, 400])):
        off, dev = offsets(lens)
        n, s, kept = sum(lens), len(lens), (0, 2)
        for value in VALUES:
            for silu, backwards in ((True, False), (False, True), (True, True)):
                p = {"x": draw(1, n, c, dtype=dtype), "w": draw(2, taps, c), "bias": draw(3, c), "before": draw(4, s, taps - 1, c), "dy": draw(5, n, c, dtype=dtype),
                     "dlast": draw(6, s, taps - 1, c)}
                if what in ("x", "dy"):
                    p[what][7, c // 2] = value
                elif what in ("before", "dlast"):
                    p[what][kept, taps // 2 - 1, c // 2] = value
                else:
                    p[what].view(-1, c)[taps // 2 if what == "w" else 0, c // 2] = value
                g = {k: t.cuda() for k, t in p.items()}
                y, last = torch.empty_like(g["x"]), torch.empty_like(g["before"])
                ctx.causal_conv(DT[dtype], g["x"], g["w"], dev, y, bias=g["bias"], silu=silu, backwards=backwards, before=g["before"], last=last)
                out = {k: torch.empty_like(g[q]) for k, q in (("dx", "x"), ("dw", "w"), ("dbias", "bias"), ("dbefore", "before"))}
                ctx.causal_conv_backward(DT[dtype], g["x"], g["w"], dev, g["dy"], out["dx"], out["dw"], work(ctx.causal_conv_work(DT[dtype], n, c, taps)),
                                         bias=g["bias"], dbias=out["dbias"], silu=silu, backwards=backwards, before=g["before"], dlast=g["dlast"],
                                         dbefore=out["dbefore"])
                e = {k: f64(t) for k, t in p.items()}
                with np.errstate(all="ignore"):
                    exp = (*V.causal_conv(e["x"], e["w"], e["bias"], off, e["before"], silu, backwards),
                           *V.causal_conv_backward(e["x"], e["w"], e["bias"], off, e["before"], e["dy"], e["dlast"], silu, backwards))
                for k, got, v in zip(("y", "last", *out), (y, last, *out.values()), exp):
                    _check(got, v, (k, c, taps, value, silu, backwards))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("what", ["x", "branch", "gate", "dsum", "dy", "post", "scale", "next"])
def test_gated_residual(ctx, dtype, what):
    n = 45
    for c in (1, 3, 9, 24, 90, 130, 1000):
        for value in VALUES:
            p = {k: draw(i, n, c, dtype=dtype) for i, k in enumerate(("x", "branch", "gate", "dsum", "dy"))}
            p.update(post=draw(6, c), scale=draw(7, 1), next=draw(8, c))
            p[what].view(-1, p[what].shape[-1])[11 if p[what].dim() == 2 else 0, 0 if what == "scale" else c // 2] = value
            g = {k: t.cuda() for k, t in p.items()}
            total, y = torch.empty_like(g["x"]), torch.empty_like(g["x"])
            ctx.gated_residual(DT[dtype], g["x"], g["branch"], g["post"], g["scale"], total, 1e-5, gate=g["gate"], next_gain=g["next"], y=y)
            out = {k: torch.empty_like(g[q]) for k, q in (("dx", "x"), ("dbranch", "x"), ("dgate", "x"), ("dpost", "post"), ("dscale", "scale"), ("dnext", "next"))}
            ctx.gated_residual_backward(DT[dtype], g["x"], g["branch"], g["post"], g["scale"], 1e-5, g["dsum"], out["dx"], out["dbranch"], out["dpost"],
                                        out["dscale"], work(ctx.gated_residual_work(DT[dtype], n, c)), gate=g["gate"], dgate=out["dgate"], next_gain=g["next"],
                                        dy=g["dy"], dnext=out["dnext"])
            e = {k: f64(t) for k, t in p.items()}
            args = e["x"], e["branch"], e["gate"], e["post"], e["scale"], e["next"], 1e-5
            with np.errstate(all="ignore"):
                es, ey = V.gated_residual(*args)
                exp = V.gated_residual_backward(*args, e["dsum"], e["dy"])
            _check(total, es, ("sum", c, value))
            _check(y, ey, ("y", c, value))
            for k in out:
                _check(out[k], exp[k], (k, c, value))
