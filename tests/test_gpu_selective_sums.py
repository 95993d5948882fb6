"""Gradients of parameters summed over long calls: the scan's against the oracle, within bounds that a lost chunk of rows would leave (test_selective_sums.py); the
convolution's where every block takes more than one turn over the rows, against the formula in 64 bits on the GPU."""
import numpy as np
import pytest
import torch

from paper_2507_04123_amd import binding as B

import selective_sums as S
from selective_bounds import E, TINY, U
from selective_helpers import DT, f64, within, work

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


@pytest.mark.parametrize("dtype,backwards", [("f32", False), ("f32", True), ("f16", False), ("bf16", True)])
def test_scan_weights(ctx, dtype, backwards):
    p = S.case(dtype)
    off = np.concatenate([[0], np.cumsum(S.LENS)])
    g, dev = {k: t.cuda() for k, t in p.items()}, torch.from_numpy(off.astype(np.int32)).cuda()
    n, (c, m) = int(off[-1]), p["a"].shape
    out = {k: torch.empty_like(g[q]) for k, q in (("dx", "x"), ("ddt", "dt"), ("da", "a"), ("db", "b"), ("dc", "c"), ("dskip", "skip"), ("ddt_bias", "dt_bias"))}
    ctx.selective_scan_backward(DT[dtype], *[g[k] for k in ("x", "dt", "a", "b", "c")], dev, g["dy"], *[out[k] for k in ("dx", "ddt", "da", "db", "dc")],
                                work(ctx.selective_scan_work(DT[dtype], n, c, m)), skip=g["skip"], dskip=out["dskip"], dt_bias=g["dt_bias"],
                                ddt_bias=out["ddt_bias"], backwards=backwards)
    e = {k: f64(t) for k, t in p.items()}
    terms, bounds = S.terms_and_bounds(*[e[k] for k in ("x", "dt", "a", "b", "c")], off, *[e[k] for k in ("h0", "skip", "dt_bias", "dy", "dlast")], backwards)
    for k in S.NAMES:
        within(out[k], terms[k].sum(0), bounds[k], k)


# A call of three channels has 85 runs of 60 rows a block and 2048 blocks at most: 10.4 million rows are one turn.  Bounds as in selective_bounds, of all rows at
# once; behind a weight's part: 60 rows a turn, seven additions by halves in the block, eight turns of the blocks' lines and eight additions by halves.
@pytest.mark.parametrize("dtype,taps,backwards", [("f16", 4, False), ("bf16", 3, True)])
def test_conv_of_more_rows_than_one_turn(ctx, dtype, taps, backwards):
    c, lens = 3, [5000000, 0, 1, 2, 3, 4000011, 0, 1500002, 900001]
    off = np.concatenate([[0], np.cumsum(lens)])
    n, dev = int(off[-1]), torch.from_numpy(off.astype(np.int32)).cuda()
    td = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    r = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    x, dy = (r(n, c).abs() + 0.25).to(td), (r(n, c).abs() + 0.25).to(td)
    w, bias, before, dlast = r(taps, c) * 0.5, r(c), r(len(lens), taps - 1, c).abs(), r(len(lens), taps - 1, c)
    y, dx = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    dw, db, dbefore = torch.full_like(w, 9.0), torch.full_like(bias, 9.0), torch.full_like(before, 9.0)
    ctx.causal_conv(DT[dtype], x, w, dev, y, bias=bias, backwards=backwards, before=before)
    ctx.causal_conv_backward(DT[dtype], x, w, dev, dy, dx, dw, work(ctx.causal_conv_work(DT[dtype], n, c, taps)), bias=bias, dbias=db, backwards=backwards,
                             before=before, dlast=dlast, dbefore=dbefore)
    turn = lambda t: t.flip(0) if backwards else t  # noqa: E731
    length = torch.from_numpy(np.diff(off)).cuda()
    length, k = turn(length), len(lens)
    first = torch.cumsum(length, 0) - length
    seq = torch.repeat_interleave(torch.arange(k, device="cuda"), length)
    row = torch.arange(n, device="cuda")
    depth, left = row - first[seq], (first + length)[seq] - 1 - row
    w64, b64, before64, dlast64 = w.double(), bias.double(), turn(before).double(), turn(dlast).double()

    def past(j):                                                         # x of j rows before every row
        v = turn(x).double()
        return torch.where((depth >= j)[:, None], v[(row - j).clamp(min=0)], before64[seq, (depth - j + taps - 1).clamp(0, taps - 2)]) if j else v

    z = b64 + sum(w64[j] * past(j) for j in range(taps))
    ez = (taps + 4) * E * (b64.abs() + sum((w64[j] * past(j)).abs() for j in range(taps)))
    on = torch.sigmoid(z)
    value, slope = z * on, on * (1 + z * (1 - on))
    tiny, u = TINY["f32"], U[dtype]

    def outside(got, exp, err):
        return int((~((turn(got).double() - exp).abs() <= err + u * (exp.abs() + err) + TINY[dtype])).sum())

    assert outside(y, value, 1.1 * ez + 16 * E * (1 + z.abs()) * value.abs() + tiny) == 0
    dyd = turn(dy).double()
    dz = dyd * slope
    edz = dyd.abs() * (0.5 * ez + 32 * E * (1 + z * z) * (slope.abs() + 0.01)) + 2 * E * dz.abs()
    blocks = min(2048, -(-n // (60 * 85)))
    turns = -(-n // (blocks * 60 * 85))
    assert turns == 2
    chain = (60 * turns + 7 + 8 + 8) * E
    del value, slope, on, ez, z
    got = [dw[j] for j in range(taps)] + [db]
    for j in range(taps + 1):
        v = past(j) if j < taps else torch.ones((), dtype=torch.float64, device="cuda")
        exp, bound = (dz * v).sum(0), ((edz + chain * dz.abs()) * v.abs()).sum(0) + tiny
        assert ((got[j].double() - exp).abs() <= bound).all(), (j, got[j], exp, bound)
        if j == taps:                                                    # a lost turn, or a thousandth of one, would show
            assert (bound < 1e-3 * dz.abs().sum(0) / 2 * (exp.abs() / dz.abs().sum(0)).clamp(min=0.05)).all()
    exp, err = torch.zeros_like(dz), torch.zeros_like(dz)
    for j in range(taps):
        there = (left >= j)[:, None]
        at = (row + j).clamp(max=n - 1)
        exp += torch.where(there, w64[j] * dz[at], 0)
        err += torch.where(there, w64[j].abs() * (edz + (taps + 4) * E * dz.abs())[at], 0)
    near = left < taps - 1                                               # the rows kept: their gradients come to them
    exp[near] += dlast64[seq[near], taps - 2 - left[near]]
    err[near] += (taps + 4) * E * dlast64[seq[near], taps - 2 - left[near]].abs()
    assert outside(dx, exp, err) == 0
    # the rows before: of each sequence's first rows, a sequence at a time
    got = turn(dbefore).double()
    for s in range(k):
        for i in range(taps - 1):
            e, b = torch.zeros(c, dtype=torch.float64, device="cuda"), torch.zeros(c, dtype=torch.float64, device="cuda") + tiny
            for j in range(taps - 1 - i, taps):
                p = i - (taps - 1) + j
                if p < int(length[s]):
                    e += w64[j] * dz[int(first[s]) + p]
                    b += w64[j].abs() * (edz + (taps + 4) * E * dz.abs())[int(first[s]) + p]
            if i - int(length[s]) >= 0:                                  # still among the rows kept
                e += dlast64[s, i - int(length[s])]
                b += (taps + 4) * E * dlast64[s, i - int(length[s])].abs()
            assert ((got[s, i] - e).abs() <= b).all(), (s, i)
