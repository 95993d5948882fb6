"""The block that runs convolution, selective scan and gated residual together: over the voxels of a backbone's level, trained, served row by row, and recorded
into a HIP graph.  Each stage is held to the oracle's on the stage's own inputs, within the bounds of the number formats."""
import numpy as np
import pytest
import torch

from oracle import selective as V
from oracle import sequence as S
from paper_2507_04123_amd import binding as B
from paper_2507_04123_amd import gen
from paper_2507_04123_amd.configs import Branch, Layer, STRIDED, SUBM, VoxelSpec
from paper_2507_04123_amd.pipeline import BranchRunner, cells_of, default_capacities, device_params
from paper_2507_04123_amd.sequence import SelectiveBlock, selective_params

import selective_bounds as L
from selective_helpers import f64, within

pytestmark = pytest.mark.gpu
NAME = {B.F32: "f32", B.F16: "f16", B.BF16: "bf16"}
TD = {B.F32: torch.float32, B.F16: torch.float16, B.BF16: torch.bfloat16}


def _block(ctx, dtype, cap, frames, c, m, taps=4, **more):
    p = selective_params(gen.make_selective_params(c, m, taps, 5))
    return SelectiveBlock(ctx, dtype, cap, frames, p, **more), {k: f64(v) for k, v in p.items()}


def _inputs(dtype, lens, b, cap, seed=1):
    r = np.random.RandomState(seed)
    off = np.concatenate([[0], np.cumsum(lens)])
    k, c, m = len(lens), b.channels, b.states
    t = {"rows": (cap, b.width), "x": (cap, c), "dtotal": (cap, c), "dy": (cap, c), "before": (k, b.taps - 1, b.inner), "h0": (k, c, m),
         "dkept": (k, b.taps - 1, b.inner), "dlast": (k, c, m)}
    t = {n: torch.from_numpy(r.standard_normal(shape)).to(TD[dtype] if len(shape) == 2 else torch.float32).cuda() for n, shape in t.items()}
    return off, torch.from_numpy(off.astype(np.int32)).cuda(), t


def _args(b, p, n, rows, off, before, h0):
    """Arguments of the stages' definitions, each of the stage's own inputs."""
    c, m = b.channels, b.states
    rows, v = f64(rows[:n]), f64(b.v[:n])
    conv = rows[:, c:c + b.inner], p["conv_w"], p["conv_bias"], off, before
    scan = v[:, :c], rows[:, c + b.inner:], p["a"], v[:, c:c + m], v[:, c + m:], off, h0, p["skip"], p["dt_bias"]
    return conv, scan, lambda x, s: (x, s, rows[:, :c], p["post"], p["scale"], p["next"], 1e-5)


def _check_run(b, p, rows, x, off, before, h0):
    name, n = NAME[b.dtype], off[-1]
    conv, scan, join = _args(b, p, n, rows, off, before, h0)
    v, kept = V.causal_conv(*conv, True, b.backwards)
    within(b.v[:n], v, L.causal_conv(*conv, True, b.backwards, name), "v")
    assert np.array_equal(f64(b.kept), kept)
    s, last = V.selective_scan(*scan, b.backwards)
    bs, bl = L.selective_scan(*scan, b.backwards, name)
    within(b.s[:n], s, bs, "s")
    within(b.last, last, bl, "last")
    args = join(f64(x[:n]), f64(b.s[:n]))
    for got, e, bound, what in zip((b.total[:n], b.y[:n]), V.gated_residual(*args), L.gated_residual(*args, name), ("total", "y")):
        within(got, e, bound, what)


@pytest.mark.parametrize("dtype", [B.F16, B.BF16])
def test_block_over_the_voxels_of_a_backbone_level(dtype):
    nb, per = 3, 2500
    spec = VoxelSpec((0.0, -10.0, -3.0), (0.2, 0.2, 0.2), (100, 100, 20), nb)
    br = Branch("b", spec, (Layer(SUBM, 4, 32), Layer(STRIDED, 32, 64)))
    pts = np.concatenate([gen.make_cloud("uniform_tiny", per, gen.frame_seed(1, i)) for i in range(nb)]).astype(np.float32)
    batch = np.repeat(np.arange(nb, dtype=np.int32), per)
    batch[batch == 1] = 2                                    # the middle frame has no points
    caps = default_capacities(br, len(pts))
    ctx = B.Context(len(pts), max(caps), cells_of(spec.grid, nb), n_slots=len(caps))
    runner = BranchRunner(ctx, br, dtype, len(pts), device_params(br.layers, 3, dtype), capacities=caps)
    feats = runner.run(torch.from_numpy(pts).cuda(), torch.from_numpy(batch).cuda())
    lv = runner.levels[-1]
    b, p = _block(ctx, dtype, lv.cap, nb, 64, 8, backwards=True)
    off = torch.zeros(nb + 1, dtype=torch.int32, device="cuda")
    ctx.frame_offsets(lv.coords, lv.n, lv.cap, nb, off)
    project = torch.from_numpy(np.random.RandomState(2).standard_normal((64, b.width)) / 8).to(TD[dtype]).cuda()
    rows = feats @ project
    b.run(rows, feats, off)
    ctx.status_sync()
    n = int(lv.n.item())
    want = S.frame_offsets(lv.coords[:n].cpu().numpy(), nb)
    assert off.tolist() == want.tolist() and want[1] == want[2] and want[3] == n > 1000
    _check_run(b, p, rows, feats, want, np.zeros((nb, 3, b.inner)), np.zeros((nb, 64, 8)))
    ctx.close()


@pytest.mark.parametrize("dtype", [B.F32, B.F16, B.BF16])
@pytest.mark.parametrize("backwards", [False, True])
def test_block_and_its_gradients_stage_by_stage(dtype, backwards):
    ctx = B.Context(1, 1, 1)
    b, p = _block(ctx, dtype, 1400, 4, 24, 6, taps=3, backwards=backwards, train=True)
    off, offsets, t = _inputs(dtype, [700, 0, 1, 430], b, 1400)
    n, name, c, m = off[-1], NAME[dtype], 24, 6
    b.run(t["rows"], t["x"], offsets, t["before"], t["h0"])
    drows, dx = b.backward(t["rows"], t["x"], offsets, t["dtotal"], t["dy"], t["before"], t["h0"], t["dkept"], t["dlast"])
    ctx.status_sync()
    _check_run(b, p, t["rows"], t["x"], off, f64(t["before"]), f64(t["h0"]))
    conv, scan, join = _args(b, p, n, t["rows"], off, f64(t["before"]), f64(t["h0"]))
    args = *join(f64(t["x"][:n]), f64(b.s[:n])), f64(t["dtotal"][:n]), f64(t["dy"][:n])
    exp, bound = V.gated_residual_backward(*args), L.gated_residual_backward(*args, name)
    got = {"dx": dx[:n], "dbranch": b.ds[:n], "dgate": drows[:n, :c], "dpost": b.grads["post"], "dscale": b.grads["scale"], "dnext": b.grads["next"]}
    for k in exp:
        within(got[k], exp[k], bound[k], k)
    args = *scan, f64(b.ds[:n]), f64(t["dlast"]), backwards
    exp, bound = V.selective_scan_backward(*args), L.selective_scan_backward(*args, name)
    got = {"dx": b.dv[:n, :c], "db": b.dv[:n, c:c + m], "dc": b.dv[:n, c + m:], "ddt": drows[:n, c + b.inner:], "da": b.grads["a"], "dskip": b.grads["skip"],
           "ddt_bias": b.grads["dt_bias"], "dh0": b.dh0}
    for k in exp:
        within(got[k], exp[k], bound[k], k)
    args = *conv, f64(b.dv[:n]), f64(t["dkept"]), True, backwards
    for got, e, bound, what in zip((drows[:n, c:c + b.inner], b.grads["conv_w"], b.grads["conv_bias"], b.dkept), V.causal_conv_backward(*args),
                                   L.causal_conv_backward(*args, name), ("dxbc", "dw", "dbias", "dkept")):
        within(got, e, bound, what)
    ctx.close()


def test_block_gradient_is_the_difference_of_its_loss():
    """fp32 gradients along random directions against central differences of the block in 64 bits.  A gradient's values are exact to about 1e-6 of the
    terms they are sums of (fp32 sums of some hundred rows, states and norms between them), the difference to 1e-8: 1e-5 of the sum of magnitudes is asked."""
    ctx = B.Context(1, 1, 1)
    b, p = _block(ctx, B.F32, 130, 3, 8, 4, train=True)
    off, offsets, t = _inputs(B.F32, [60, 0, 70], b, 130)
    b.run(t["rows"], t["x"], offsets, t["before"], t["h0"])
    drows, dx = b.backward(t["rows"], t["x"], offsets, t["dtotal"], t["dy"], t["before"], t["h0"], t["dkept"], t["dlast"])
    c, m = 8, 4

    def loss(a):
        rows = a["rows"]
        v, kept = V.causal_conv(rows[:, c:c + b.inner], a["conv_w"], a["conv_bias"], off, a["before"])
        s, last = V.selective_scan(v[:, :c], rows[:, c + b.inner:], a["a"], v[:, c:c + m], v[:, c + m:], off, a["h0"], a["skip"], a["dt_bias"])
        total, y = V.gated_residual(a["x"], s, rows[:, :c], a["post"], a["scale"], a["next"], 1e-5)
        return sum((q * f64(t[d])).sum() for q, d in ((total, "dtotal"), (y, "dy"), (kept, "dkept"), (last, "dlast")))

    at = {**p, **{k: f64(t[k]) for k in ("rows", "x", "before", "h0")}}
    grads = {**{k: f64(v) for k, v in b.grads.items()}, "rows": f64(drows), "x": f64(dx), "before": f64(b.dkept), "h0": f64(b.dh0)}
    for i, k in enumerate(at):
        d = np.random.RandomState(i).standard_normal(at[k].shape)
        num = (loss({**at, k: at[k] + 1e-5 * d}) - loss({**at, k: at[k] - 1e-5 * d})) / 2e-5
        assert abs(num - (grads[k] * d).sum()) <= 1e-5 * np.abs(grads[k] * d).sum() + 1e-6 * (1 + abs(num)), k
    ctx.close()


@pytest.mark.parametrize("train", [False, True])
def test_block_step_moves_on_where_a_run_ended_and_changes_no_gradient(train):
    ctx = B.Context(1, 1, 1)
    frames = 5
    b, p = _block(ctx, B.F16, 200, frames, 32, 16, train=train)
    off, offsets, t = _inputs(B.F16, [40] * frames, b, 200)

    def gradients():
        drows, dx = b.backward(t["rows"], t["x"], offsets, t["dtotal"], t["dy"], t["before"], t["h0"])
        return [q.clone() for q in (drows, dx, b.dkept, b.dh0, *b.grads.values())]

    b.run(t["rows"], t["x"], offsets, t["before"], t["h0"])
    expected = gradients() if train else []
    b.run(t["rows"], t["x"], offsets, t["before"], t["h0"])
    kept, h = b.kept.clone(), b.last.clone()
    for i in range(3):
        _, _, new = _inputs(B.F16, [1] * frames, b, frames, seed=10 + i)
        one, before, h0 = np.arange(frames + 1), f64(kept), f64(h)
        c, m = b.channels, b.states
        y = b.step(new["rows"], new["x"], kept, h)
        rows, v, s = f64(new["rows"]), f64((b.dv if train else b.v)[:frames]), f64((b.ds if train else b.s)[:frames])
        conv = rows[:, c:c + b.inner], p["conv_w"], p["conv_bias"], one, before
        ev, ek = V.causal_conv(*conv)
        within((b.dv if train else b.v)[:frames], ev, L.causal_conv(*conv, True, False, "f16"), "v")
        assert np.array_equal(f64(kept), ek)
        scan = v[:, :c], rows[:, c + b.inner:], p["a"], v[:, c:c + m], v[:, c + m:], one, h0, p["skip"], p["dt_bias"]
        es, eh = V.selective_scan(*scan)
        bs, bh = L.selective_scan(*scan, False, "f16")
        within((b.ds if train else b.s)[:frames], es, bs, "s")
        within(h, eh, bh, "h")
        args = f64(new["x"]), s, rows[:, :c], p["post"], p["scale"], p["next"], 1e-5
        within(y, V.gated_residual(*args)[1], L.gated_residual(*args, "f16")[1], "y")
    if train:
        assert all(torch.equal(q, r) for q, r in zip(expected, gradients()))
    ctx.close()


def test_block_recorded_into_a_graph():
    ctx = B.Context(1, 1, 1)
    b, _ = _block(ctx, B.BF16, 20000, 3, 64, 16, train=True)
    off, offsets, t = _inputs(B.BF16, [9000, 0, 11000], b, 20000)

    def both():
        b.run(t["rows"], t["x"], offsets, t["before"], t["h0"])
        b.backward(t["rows"], t["x"], offsets, t["dtotal"], t["dy"], t["before"], t["h0"], t["dkept"], t["dlast"])

    results = lambda: (b.y, b.total, b.kept, b.last, b.drows, b.dx, b.dkept, b.dh0, *b.grads.values())  # noqa: E731
    both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        t["rows"].normal_(generator=torch.Generator(device="cuda").manual_seed(i))
        both()
        torch.cuda.synchronize()
        kept = [q.clone() for q in results()]
        for q in (*results(), b.v, b.s, b.dv, b.ds):
            q.zero_()
        b.work.fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(kept, results()))
    ctx.status_sync()
    ctx.close()


def test_block_refuses_what_it_was_not_made_for():
    ctx = B.Context(1, 1, 1)
    b, _ = _block(ctx, B.F16, 16, 1, 16, 4)
    off, offsets, t = _inputs(B.F16, [16], b, 16)
    b.run(t["rows"], t["x"], offsets)
    with pytest.raises(ValueError, match="train"):
        b.backward(t["rows"], t["x"], offsets, None, t["dy"])
    with pytest.raises(ValueError, match="values a row"):
        b.run(t["rows"][:, 1:], t["x"], offsets)
    with pytest.raises(ValueError, match="parameters"):
        b.load({**b.params, "a": b.params["a"][:, :2].contiguous()})
    ctx.close()
