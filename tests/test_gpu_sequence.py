"""The sequence operators (layer norm, gated linear recurrence, gated feed-forward network) against the oracle in 64 bits, within the
bounds that the number formats give; their refusals."""
import itertools

import numpy as np
import pytest
import torch

from oracle import sequence as S
from paper_2507_04123_amd import binding as B

import sequence_bounds as L

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DT = {"f32": B.F32, "f16": B.F16, "bf16": B.BF16}
TYPES = list(TD)


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


def _draw(seed, *shape, scale=1.0, shift=0.0, dtype="f32"):
    v = torch.from_numpy(np.random.RandomState(seed).standard_normal(shape) * scale + shift)
    return v.to(TD[dtype])


def _np(t):
    return t.double().cpu().numpy()


def _rows(t, how):
    """The rows `t` on the GPU: packed; a 16-byte aligned slice of wider rows; an odd slice of them."""
    t = t.cuda()
    if how == "packed":
        return t
    n, c = t.shape
    at = 16 if how == "slice" else 1
    wide = torch.full((n, (c + 2 * at + 15) // 16 * 16 + (0 if how == "slice" else 3)), 7.0, dtype=t.dtype, device="cuda")
    wide[:, at:at + c] = t
    return wide[:, at:at + c]


def _like(t, how):
    return _rows(torch.full(t.shape, -3.0, dtype=t.dtype), how)


def _within(got, exp, bound, what):
    got = _np(got)
    assert got.shape == exp.shape, what
    bad = ~(np.abs(got - exp) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside, first {i}: {got[i]!r}, {exp[i]!r} +- {bound[i]:.3g}")


def _work(size):
    return torch.full((max(size, 16),), 0xA5, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------------------ layer norm

WIDTHS = [1, 3, 8, 16, 47, 64, 90, 128, 160, 250, 384, 511, 512, 1000, 1024]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", WIDTHS)
def test_layernorm(ctx, dtype, c):
    for rows, how in ((1, "packed"), (37, "slice"), (301, "odd"), (64, "packed")):
        x = _draw(c, rows, c, scale=2.0, shift=1.0, dtype=dtype)
        x[rows // 2] = 0
        res = _draw(c + 1, rows, c, dtype=dtype)
        gamma, beta = _draw(c + 2, c, scale=0.3, shift=1.0), _draw(c + 3, c)
        x_, res_, y, total = _rows(x, how), _rows(res, how), _like(x, how), _like(x, how)
        ctx.layernorm(DT[dtype], x_, gamma.cuda(), beta.cuda(), 1e-5, y)
        xs, g, b = _np(x), _np(gamma), _np(beta)
        _within(y, S.layernorm(xs, g, b, 1e-5), L.layernorm(xs, g, b, 1e-5, dtype), "y")
        ctx.layernorm(DT[dtype], x_, gamma.cuda(), beta.cuda(), 1e-5, y, residual=res_, total=total)
        # the sum in fp32 (one rounding), then as above of what that is
        s = _np(x.float() + res.float())
        _within(total, s, L.rounded(s, 0.0, dtype), "sum")
        _within(y, S.layernorm(s, g, b, 1e-5), L.layernorm(s, g, b, 1e-5, dtype), "y of the sum")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", WIDTHS)
def test_layernorm_backward(ctx, dtype, c):
    for rows, how, with_add in ((1, "packed", False), (37, "slice", True), (700, "odd", True), (1200, "packed", False)):
        x, dy, add = _draw(c, rows, c, scale=2.0, shift=1.0, dtype=dtype), _draw(c + 1, rows, c, dtype=dtype), _draw(c + 2, rows, c, dtype=dtype)
        x[rows // 2] = 0
        gamma = _draw(c + 3, c, scale=0.3, shift=1.0)
        dx, dg, db = _like(x, how), torch.full((c,), 9.0, device="cuda"), torch.full((c,), 9.0, device="cuda")
        ctx.layernorm_backward(DT[dtype], _rows(x, how), gamma.cuda(), 1e-5, _rows(dy, how), dx, dg, db,
                               _work(ctx.layernorm_work(DT[dtype], rows, c)), add=_rows(add, how) if with_add else None)
        xs, g, d, ad = _np(x), _np(gamma), _np(dy), _np(add) * with_add
        ex, eg, eb = S.layernorm_backward(xs, g, 1e-5, d)
        bx, bg, bb = L.layernorm_backward(xs, g, 1e-5, d, ad, dtype)
        _within(dx, ex + ad, bx, "dx")
        _within(dg, eg, bg, "dgamma")
        _within(db, eb, bb, "dbeta")


@pytest.mark.parametrize("dtype", TYPES)
def test_layernorm_device_count_in_place_and_no_rows(ctx, dtype):
    c, cap = 64, 50
    x, dy, gamma, beta = _draw(1, cap, c, dtype=dtype).cuda(), _draw(2, cap, c, dtype=dtype).cuda(), torch.ones(c).cuda(), torch.zeros(c).cuda()
    whole = torch.empty_like(x)
    ctx.layernorm(DT[dtype], x, gamma, beta, 1e-5, whole)
    for n in (0, 1, 33, 50, 99, -4):
        rows = min(max(n, 0), cap)
        y, count = x.clone(), torch.tensor([n], dtype=torch.int32, device="cuda")
        ctx.layernorm(DT[dtype], y, gamma, beta, 1e-5, y, n=count)                  # in place
        assert torch.equal(y[:rows], whole[:rows]) and torch.equal(y[rows:], x[rows:])
        poison = x.clone()
        poison[rows:] = float("nan")                                                # rows beyond the count are not looked at
        out = []
        for cap_ in (cap, rows):
            dx, dg, db = torch.zeros_like(x), torch.full((c,), 9.0, device="cuda"), torch.full((c,), 9.0, device="cuda")
            ctx.layernorm_backward(DT[dtype], poison[:cap_], gamma, 0.0 if n == 33 else 1e-5, dy[:cap_], dx[:cap_], dg, db,
                                   _work(ctx.layernorm_work(DT[dtype], cap, c)), n=count if cap_ == cap else None)
            out.append((dx, dg, db))
        assert all(torch.isfinite(t).all() for t in out[0]) and torch.equal(out[0][0], out[1][0])
        if rows == 0:
            assert not out[0][1].any() and not out[0][2].any() and not out[1][1].any() and not out[1][2].any()


# ------------------------------------------------------------------------------------------------------------ recurrence

LENGTHS = {"one": [1], "none": [0], "empties": [0, 5, 0, 0, 7, 1, 0], "tile": [256], "long": [3000], "around": [255, 1, 256, 257, 0, 511],
           "short": [3, 0, 1, 2, 9, 4] * 60, "ragged": [1, 700, 0, 33, 1500, 2, 64, 64]}


def _sequences(name, c, dtype, seed):
    lens = LENGTHS[name]
    off = np.concatenate([[0], np.cumsum(lens)])
    n = int(off[-1])
    x, gate = _draw(seed, n, c, dtype=dtype), _draw(seed + 1, n, c, scale=2.0, shift=1.5, dtype=dtype)
    gate[::11] *= 8
    return off, x, gate, _draw(seed + 2, len(lens), c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("backwards", [False, True])
def test_recurrence(ctx, dtype, name, backwards):
    for c, how, state in ((64, "packed", True), (96, "slice", True), (7, "odd", False), (16, "packed", False), (100, "odd", True)):
        off, x, gate, h0 = _sequences(name, c, dtype, c)
        dy, dlast = _draw(90, len(x), c, dtype=dtype), _draw(91, *h0.shape)
        offsets = torch.from_numpy(off.astype(np.int32)).cuda()
        work = _work(ctx.recurrence_work(DT[dtype], len(x), c))
        x_, gate_, y, last = _rows(x, how), _rows(gate, how), _like(x, how), torch.full(h0.shape, 5.0, device="cuda")
        h_ = h0.cuda() if state else None
        ctx.recurrence(DT[dtype], x_, gate_, offsets, y, work, backwards=backwards, h0=h_, last=last)
        xs, gs, hs, ds, ls = _np(x), _np(gate), _np(h0) * state, _np(dy), _np(dlast) * state
        ey, el = S.recurrence(xs, gs, off, hs, backwards)
        by, bl, _ = L.recurrence(xs, gs, off, hs, backwards, dtype)
        _within(y, ey, by, f"y {c}")
        _within(last, el, bl, f"last {c}")
        dx, dg, dh0 = _like(x, how), _like(x, how), torch.full(h0.shape, 5.0, device="cuda")
        ctx.recurrence_backward(DT[dtype], x_, gate_, offsets, _rows(dy, how), dx, dg, work, backwards=backwards, h0=h_,
                                dlast=dlast.cuda() if state else None, dh0=dh0)
        exp = S.recurrence_backward(xs, gs, off, hs, ds, ls, backwards)
        for got, e, b, what in zip((dx, dg, dh0), exp, L.recurrence_backward(xs, gs, off, hs, ds, ls, backwards, dtype), ("dx", "dgate", "dh0")):
            _within(got, e, b, f"{what} {c}")


@pytest.mark.parametrize("backwards", [False, True])
def test_recurrence_keeps_infinities_and_nan_to_their_sequence_and_channel(ctx, backwards):
    for name, c in itertools.product(("around", "short", "ragged"), (64, 5)):
        off, x, gate, h0 = _sequences(name, c, "f32", 3)
        dy, dlast = _draw(4, len(x), c), _draw(5, *h0.shape)
        offsets, bad = torch.from_numpy(off.astype(np.int32)).cuda(), [s for s in range(len(off) - 1) if off[s + 1] > off[s]][1::3]
        work = _work(ctx.recurrence_work(B.F32, len(x), c))

        def run(x, gate, h0, dy):
            out = [torch.zeros_like(x), torch.zeros_like(h0), torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(h0)]
            ctx.recurrence(B.F32, x, gate, offsets, out[0], work, backwards=backwards, h0=h0, last=out[1])
            ctx.recurrence_backward(B.F32, x, gate, offsets, dy, out[2], out[3], work, backwards=backwards, h0=h0, dlast=dlast.cuda(), dh0=out[4])
            return out

        clean = run(x.cuda(), gate.cuda(), h0.cuda(), dy.cuda())
        for what, value in itertools.product(range(4), (float("inf"), float("nan"))):
            args = [t.clone() for t in (x, gate, h0, dy)]
            for s in bad:
                args[what][s if what == 2 else (off[s] + off[s + 1] - 1) // 2, 2] = value
            dirty = run(*(t.cuda() for t in args))
            rows, seqs = torch.ones(len(x), dtype=torch.bool), torch.ones(len(h0), dtype=torch.bool)
            for s in bad:
                rows[off[s]:off[s + 1]] = False
                seqs[s] = False
            for i, (p, q) in enumerate(zip(clean, dirty)):
                keep = (seqs if i in (1, 4) else rows).cuda()
                assert torch.equal(p[keep], q[keep]), (name, c, what, value, i)
                rest = [k for k in range(c) if k != 2]
                assert torch.equal(p[:, rest], q[:, rest]), (name, c, what, value, i)
            assert not torch.equal(clean[0], dirty[0]) or what == 3 or value == float("inf")


def test_recurrence_gates_shut_and_open(ctx):
    x, h0 = _draw(1, 600, 64).cuda(), _draw(2, 1, 64).cuda()
    off, work = torch.tensor([0, 600], dtype=torch.int32, device="cuda"), _work(ctx.recurrence_work(B.F32, 600, 64))
    for g, exp in ((200.0, h0.expand(600, 64)), (-200.0, x), (float("inf"), h0.expand(600, 64)), (float("-inf"), x)):
        y, last = torch.empty_like(x), torch.empty_like(h0)
        ctx.recurrence(B.F32, x, torch.full_like(x, g), off, y, work, h0=h0, last=last)
        assert torch.equal(y, exp) and torch.equal(last, exp[-1:])


def test_recurrence_more_rows_than_capacity_are_reported_and_left_out(ctx):
    off, x, gate, h0 = _sequences("ragged", 64, "f32", 8)
    n, cap = len(x), 900
    offsets, work = torch.from_numpy(off.astype(np.int32)).cuda(), _work(ctx.recurrence_work(B.F32, n, 64))
    for rows in (cap, 1, 5):
        cut = np.minimum(off, rows)
        y, last = torch.full((n, 64), 4.0, device="cuda"), torch.empty_like(h0).cuda()
        ctx.recurrence(B.F32, x.cuda()[:rows], gate.cuda()[:rows], offsets, y[:rows], work, h0=h0.cuda(), last=last)
        with pytest.raises(B.Emc2Error) as ei:
            ctx.status_sync()
        assert ei.value.status == B.ERR_CAPACITY
        xs, gs, hs = _np(x[:rows]), _np(gate[:rows]), _np(h0)
        ey, _ = S.recurrence(xs, gs, cut, hs)
        _within(y[:rows], ey, L.recurrence(xs, gs, cut, hs, False, "f32")[0], "y")
        assert bool((y[rows:] == 4.0).all())
    y = torch.full((n + 9, 64), 4.0, device="cuda")                                 # fewer rows than the buffers hold
    pad = torch.full((9, 64), float("nan"))
    ctx.recurrence(B.F32, torch.cat([x, pad]).cuda(), torch.cat([gate, pad]).cuda(), offsets, y, _work(ctx.recurrence_work(B.F32, n + 9, 64)),
                   h0=h0.cuda())
    ctx.status_sync()
    assert bool((y[n:] == 4.0).all()) and bool(torch.isfinite(y).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_recurrence_step_is_a_sequence_of_one(ctx, dtype):
    for rows, c, how in ((1, 8, "packed"), (8, 128, "slice"), (33, 47, "odd"), (1000, 64, "packed")):
        x, gate, h0 = _draw(1, rows, c, dtype=dtype), _draw(2, rows, c, scale=3.0, dtype=dtype), _draw(3, rows, c)
        y, h = _like(x, how), h0.cuda()
        ctx.recurrence_step(DT[dtype], _rows(x, how), _rows(gate, how), h, h, y)     # the states in place
        off = np.arange(rows + 1)
        xs, gs, hs = _np(x), _np(gate), _np(h0)
        ey, el = S.recurrence(xs, gs, off, hs)
        by, bl, _ = L.recurrence(xs, gs, off, hs, False, dtype)
        _within(y, ey, by, "y")
        _within(h, el, bl, "h")


# ------------------------------------------------------------------------------------------------------------ feed-forward

SIZES = [(1, 1), (8, 32), (32, 31), (33, 100), (48, 200), (64, 256), (90, 64), (96, 96), (128, 512), (151, 177), (160, 320), (192, 64), (200, 33),
         (256, 300)]


def _weights(c, f, dtype):
    return [_draw(c + i, *s, scale=s[0] ** -0.5, dtype=dtype) for i, s in enumerate(((c, f), (c, f), (f, c)))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c,f", SIZES)
def test_ffn_and_its_gradients(ctx, dtype, c, f):
    w = _weights(c, f, dtype)
    packed = torch.full((ctx.ffn_packed_size(DT[dtype], c, f),), float("nan"), dtype=TD[dtype], device="cuda")
    ctx.ffn_pack(DT[dtype], *(t.cuda() for t in w), packed)
    wg, wu, wd = (_np(t) for t in w)
    for rows, how, act in ((1, "packed", "silu"), (33, "odd", "gelu"), (130, "slice", "silu"), (515, "packed", "gelu")):
        code = B.ACT_SILU if act == "silu" else B.ACT_GELU
        x, res, dy = (_draw(50 + i, rows, c, dtype=dtype) for i in range(3))
        y, x_ = _like(x, how), _rows(x, how)
        xs, rs, ds = _np(x), _np(res), _np(dy)
        for r in (None, res):
            ctx.ffn(DT[dtype], code, x_, packed, f, y, residual=None if r is None else _rows(r, how))
            zero = np.zeros_like(rs) if r is None else rs
            _within(y, S.ffn(act, xs, wg, wu, wd) + zero, L.ffn(act, xs, wg, wu, wd, zero, dtype), f"y {rows}")
        dx, g = _like(x, how), [torch.full(t.shape, 9.0, dtype=TD[dtype], device="cuda") for t in w]
        ctx.ffn_backward(DT[dtype], code, x_, packed, f, _rows(dy, how), dx, *g, _work(ctx.ffn_work(DT[dtype], rows, c, f)))
        for got, e, b, what in zip((dx, *g), S.ffn_backward(act, xs, wg, wu, wd, ds), L.ffn_backward(act, xs, wg, wu, wd, ds, dtype),
                                   ("dx", "dwg", "dwu", "dwd")):
            _within(got, e, b, f"{what} {rows}")


@pytest.mark.parametrize("dtype", TYPES)
def test_ffn_many_rows_device_count_in_place_and_no_rows(ctx, dtype):
    c, f, cap = 64, 96, 9000
    w = _weights(c, f, dtype)
    packed = torch.empty(ctx.ffn_packed_size(DT[dtype], c, f), dtype=TD[dtype], device="cuda")
    ctx.ffn_pack(DT[dtype], *(t.cuda() for t in w), packed)
    x, dy = _draw(1, cap, c, dtype=dtype).cuda(), _draw(2, cap, c, dtype=dtype).cuda()
    whole, work = torch.empty_like(x), _work(ctx.ffn_work(DT[dtype], cap, c, f))
    ctx.ffn(DT[dtype], B.ACT_SILU, x, packed, f, whole)
    for n in (0, 1, 31, 4097, cap, cap + 5):
        rows, count = min(n, cap), torch.tensor([n], dtype=torch.int32, device="cuda")
        y = x.clone()
        ctx.ffn(DT[dtype], B.ACT_SILU, y, packed, f, y, n=count)                      # in place
        assert torch.equal(y[:rows], whole[:rows]) and torch.equal(y[rows:], x[rows:])
        poison, flow = x.clone(), dy.clone()
        poison[rows:], flow[rows:] = float("nan"), float("nan")
        g = [torch.full(t.shape, 9.0, dtype=TD[dtype], device="cuda") for t in w]
        ctx.ffn_backward(DT[dtype], B.ACT_SILU, poison, packed, f, flow, flow, *g, work, n=count)   # dx where dy lies
        assert bool(torch.isnan(flow[rows:]).all()) and all(bool(torch.isfinite(t).all()) for t in (flow[:rows], *g))
        xs, ds, ws = _np(x[:rows]), _np(dy[:rows]), [_np(t) for t in w]
        if rows:
            for got, e, b in zip((flow[:rows], *g), S.ffn_backward("silu", xs, *ws, ds), L.ffn_backward("silu", xs, *ws, ds, dtype)):
                _within(got, e, b, f"gradient {n}")
        else:
            assert not any(t.any() for t in g)
    g = [torch.full(t.shape, 9.0, dtype=TD[dtype], device="cuda") for t in w]
    ctx.ffn_backward(DT[dtype], B.ACT_SILU, x[:0], packed, f, dy[:0], dy[:0].clone(), *g, work)
    ctx.ffn(DT[dtype], B.ACT_SILU, x[:0], packed, f, dy[:0])
    assert not any(t.any() for t in g)


@pytest.mark.parametrize("dtype,c", [("f16", 24), ("f16", 40), ("f16", 96), ("f16", 128), ("f16", 192), ("f16", 250), ("bf16", 64), ("bf16", 100),
                                     ("bf16", 256), ("f32", 32), ("f32", 48), ("f32", 96), ("f32", 126), ("f32", 200)])
def test_ffn_of_more_rows_than_the_chip_holds_at_once(ctx, dtype, c):
    """33 001 rows: every wave of either pass has rows of its own, and several tiles of them in the weights' gradients."""
    n, f, act, how = 33001, 72, "gelu" if c % 3 else "silu", "slice" if c % 2 else "odd" if c % 5 == 0 else "packed"
    code, w = B.ACT_SILU if act == "silu" else B.ACT_GELU, _weights(c, f, dtype)
    packed = torch.full((ctx.ffn_packed_size(DT[dtype], c, f),), float("nan"), dtype=TD[dtype], device="cuda")
    ctx.ffn_pack(DT[dtype], *(t.cuda() for t in w), packed)
    x, dy = (_draw(60 + i, n, c, dtype=dtype) for i in range(2))
    (xs, ds), ws = (_np(x), _np(dy)), [_np(t) for t in w]
    y, dx, g = _like(x, how), _like(x, how), [torch.full(t.shape, 9.0, dtype=TD[dtype], device="cuda") for t in w]
    ctx.ffn(DT[dtype], code, _rows(x, how), packed, f, y)
    _within(y, S.ffn(act, xs, *ws), L.ffn(act, xs, *ws, np.zeros_like(xs), dtype), "y")
    ctx.ffn_backward(DT[dtype], code, _rows(x, how), packed, f, _rows(dy, how), dx, *g, _work(ctx.ffn_work(DT[dtype], n, c, f)))
    for got, e, b, what in zip((dx, *g), S.ffn_backward(act, xs, *ws, ds), L.ffn_backward(act, xs, *ws, ds, dtype), ("dx", "dwg", "dwu", "dwd")):
        _within(got, e, b, what)


# ------------------------------------------------------------------------------------------------------------ all of them

def test_rows_beyond_32_bits_of_elements(ctx):
    """4 200 rows 2^20 + 8 values apart: the last ones lie beyond 2^32 elements."""
    n, c, pitch = 4200, 64, (1 << 20) + 8
    buffer = torch.empty(n * pitch, dtype=torch.float16, device="cuda")
    far = buffer.as_strided((n, c), (pitch, 1))
    x, gate = _draw(1, n, c, dtype="f16").cuda(), _draw(2, n, c, scale=2.0, shift=1.0, dtype="f16").cuda()
    gamma, beta, off = torch.ones(c).cuda(), torch.zeros(c).cuda(), torch.tensor([0, 1700, n], dtype=torch.int32, device="cuda")
    w = _weights(c, 64, "f16")
    packed = torch.empty(ctx.ffn_packed_size(B.F16, c, 64), dtype=torch.float16, device="cuda")
    ctx.ffn_pack(B.F16, *(t.cuda() for t in w), packed)
    work = _work(max(ctx.recurrence_work(B.F16, n, c), ctx.ffn_work(B.F16, n, c, 64), ctx.layernorm_work(B.F16, n, c)))

    def forward(x, y):
        ctx.layernorm(B.F16, x, gamma, beta, 1e-5, y)
        ctx.ffn(B.F16, B.ACT_SILU, y, packed, 64, y)
        ctx.recurrence(B.F16, y, gate, off, y, work)

    def backward(x, dy, dx):
        g = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in w] + [torch.empty(c, device="cuda") for _ in range(2)]
        dgate = torch.empty_like(gate)
        ctx.recurrence_backward(B.F16, x, gate, off, dy, dx, dgate, work)
        ctx.ffn_backward(B.F16, B.ACT_SILU, x, packed, 64, dx, dx, *g[:3], work)
        ctx.layernorm_backward(B.F16, x, gamma, 1e-5, dx, dx, g[3], g[4], work)
        return [dgate] + g

    near = torch.empty_like(x)
    forward(x, near)
    far.copy_(x)
    forward(far, far)
    assert torch.equal(far, near)
    one, far_dx = torch.empty_like(x), far
    exp = backward(x, near, one)
    far_dx.copy_(near)
    got = backward(x, far_dx, far_dx)
    assert torch.equal(far_dx, one) and all(torch.equal(p, q) for p, q in zip(exp, got))


def test_equal_inputs_give_equal_bits_on_other_streams(ctx):
    n, c, f = 40000, 64, 128
    x, gate, dy = (_draw(i, n, c, dtype="bf16").cuda() for i in range(3))
    off = torch.tensor([0, 10, 10, 21000, n], dtype=torch.int32, device="cuda")
    gamma, beta, w = torch.ones(c).cuda(), torch.zeros(c).cuda(), [t.cuda() for t in _weights(c, f, "bf16")]
    torch.cuda.synchronize()

    def run():
        work = _work(max(ctx.recurrence_work(B.BF16, n, c), ctx.ffn_work(B.BF16, n, c, f), ctx.layernorm_work(B.BF16, n, c)))
        packed = torch.empty(ctx.ffn_packed_size(B.BF16, c, f), dtype=torch.bfloat16, device="cuda")
        o = [torch.empty_like(x) for _ in range(7)] + [torch.empty_like(t) for t in w] + [torch.empty_like(gamma) for _ in range(2)]
        ctx.ffn_pack(B.BF16, *w, packed)
        ctx.layernorm(B.BF16, x, gamma, beta, 1e-5, o[0])
        ctx.ffn(B.BF16, B.ACT_GELU, o[0], packed, f, o[1], residual=x)
        ctx.recurrence(B.BF16, o[1], gate, off, o[2], work)
        ctx.recurrence_backward(B.BF16, o[1], gate, off, dy, o[3], o[4], work)
        ctx.ffn_backward(B.BF16, B.ACT_GELU, o[0], packed, f, o[3], o[5], *o[7:10], work)
        ctx.layernorm_backward(B.BF16, x, gamma, 1e-5, o[5], o[6], o[10], o[11], work, add=o[3])
        return o

    streams, outs = [torch.cuda.Stream() for _ in range(3)], []
    for s in streams:
        with torch.cuda.stream(s):
            outs.append(run())
    torch.cuda.synchronize()
    first = run()
    for o in outs:
        assert all(torch.equal(p, q) for p, q in zip(first, o))


@pytest.mark.parametrize("dtype", TYPES)
def test_scratch_of_the_largest_call_serves_the_smaller_ones(ctx, dtype):
    c, f, cap = 40, 200, 60000
    x, gate, dy = (_draw(i, cap, c, dtype=dtype).cuda() for i in range(3))
    gamma, w = torch.ones(c).cuda(), [t.cuda() for t in _weights(c, f, dtype)]
    packed = torch.empty(ctx.ffn_packed_size(DT[dtype], c, f), dtype=TD[dtype], device="cuda")
    ctx.ffn_pack(DT[dtype], *w, packed)

    def run(n, work):
        x_, gate_, dy_, off = x[:n], gate[:n], dy[:n], torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda")
        o = [torch.empty_like(x_) for _ in range(5)] + [torch.empty_like(t) for t in w] + [torch.empty_like(gamma) for _ in range(2)]
        ctx.recurrence(DT[dtype], x_, gate_, off, o[0], work(ctx.recurrence_work))
        ctx.recurrence_backward(DT[dtype], x_, gate_, off, dy_, o[1], o[2], work(ctx.recurrence_work))
        ctx.ffn_backward(DT[dtype], B.ACT_SILU, x_, packed, f, dy_, o[3], *o[5:8], work(ctx.ffn_work, f))
        ctx.layernorm_backward(DT[dtype], x_, gamma, 1e-5, dy_, o[4], o[8], o[9], work(ctx.layernorm_work))
        return o

    for n in (cap - 1, 33000, 16385, 8193, 700, 1):
        large = run(n, lambda query, *hidden: _work(query(DT[dtype], cap, c, *hidden)))
        own = run(n, lambda query, *hidden: _work(query(DT[dtype], n, c, *hidden)))
        assert all(torch.equal(p, q) for p, q in zip(large, own)), n


def test_frame_offsets(ctx):
    for lens in ([5, 0, 3], [0], [0, 0, 4000, 1, 0], [1] * 700):
        ids = np.repeat(np.arange(len(lens)), lens)
        coords = torch.from_numpy(np.stack([ids] + [np.zeros_like(ids)] * 3, axis=1).astype(np.int32))
        cap = len(ids) + 6
        buf = torch.full((cap, 4), 77, dtype=torch.int32)
        buf[: len(ids)] = coords
        off = torch.full((len(lens) + 1,), -1, dtype=torch.int32, device="cuda")
        ctx.frame_offsets(buf.cuda(), torch.tensor([len(ids)], dtype=torch.int32, device="cuda"), cap, len(lens), off)
        assert off.tolist() == S.frame_offsets(coords.numpy(), len(lens)).tolist()


def _raises(f, status=None):
    with pytest.raises(B.Emc2Error if status else ValueError) as ei:
        f()
    if status:
        assert ei.value.status == status


def test_refusals(ctx):
    n, c, f = 20, 64, 96
    x, g1 = torch.zeros((n, c), dtype=torch.float16, device="cuda"), torch.ones(c, device="cuda")
    y, off = torch.empty_like(x), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    work = _work(1 << 22)
    packed = torch.zeros(ctx.ffn_packed_size(B.F16, c, f), dtype=torch.float16, device="cuda")
    w = [torch.zeros(s, dtype=torch.float16, device="cuda") for s in ((c, f), (c, f), (f, c))]
    wide = torch.zeros((4, 1025), dtype=torch.float16, device="cuda")
    gw = torch.ones(1025, device="cuda")
    # another type, place, shape or stride than the call needs
    for bad in (x.float(), x.cpu(), x[:, :32], x.t().contiguous().t(), x[0]):
        _raises(lambda: ctx.layernorm(B.F16, x, g1, g1, 1e-5, bad))
        _raises(lambda: ctx.recurrence(B.F16, x, bad, off, y, work))
        _raises(lambda: ctx.recurrence_step(B.F16, x, bad, x.float(), x.float(), y))
        _raises(lambda: ctx.ffn(B.F16, B.ACT_SILU, x, packed, f, bad))
    _raises(lambda: ctx.layernorm(B.F16, x, g1[:32], g1, 1e-5, y))
    _raises(lambda: ctx.layernorm(B.F16, x, g1, g1.half(), 1e-5, y))
    _raises(lambda: ctx.layernorm_backward(B.F16, x, g1, 1e-5, x, y, g1.clone(), g1.clone(), work[:8]))
    _raises(lambda: ctx.layernorm(B.F16, x, g1, g1, 1e-5, y, n=torch.zeros(1, device="cuda")))
    big = torch.zeros((4000, c), dtype=torch.float16, device="cuda")
    _raises(lambda: ctx.recurrence(B.F16, big, big, off, big.clone(), work[:8]))
    _raises(lambda: ctx.recurrence(B.F16, x, x, off.long(), y, work))
    _raises(lambda: ctx.recurrence(B.F16, x, x, off, y, work, h0=torch.zeros((2, c), device="cuda")))
    _raises(lambda: ctx.ffn(B.F16, B.ACT_SILU, x, packed[:-1], f, y))
    _raises(lambda: ctx.ffn_pack(B.F16, w[0], w[1], w[0], packed))
    _raises(lambda: ctx.ffn_backward(B.F16, B.ACT_SILU, x, packed, f, x, y, *(torch.empty_like(t) for t in w), work[:64]))
    # sizes and values that the library itself refuses
    _raises(lambda: ctx.layernorm(B.F16, wide, gw, gw, 1e-5, wide), B.ERR_UNSUPPORTED)
    _raises(lambda: ctx.layernorm(B.F16, x, g1, g1, -1.0, y), B.ERR_INVALID_ARG)
    _raises(lambda: ctx.layernorm(B.F16, x, g1, g1, float("nan"), y), B.ERR_INVALID_ARG)
    _raises(lambda: ctx.layernorm(B.F16, x, g1, g1, 1e-5, y, total=y), B.ERR_INVALID_ARG)
    _raises(lambda: ctx.recurrence(B.F16, x, x, off[:1], y, work), B.ERR_INVALID_ARG)
    _raises(lambda: ctx.ffn(B.F16, 2, x, packed, f, y), B.ERR_INVALID_ARG)
    _raises(lambda: ctx.ffn(B.F16, B.ACT_SILU, torch.zeros((4, 257), dtype=torch.float16, device="cuda"), packed, f,
                            torch.zeros((4, 257), dtype=torch.float16, device="cuda")), B.ERR_UNSUPPORTED)
    assert ctx.ffn_packed_size(B.F16, 257, 32) == -1 and ctx.ffn_work(B.I8, 1, 1, 1) == -1 and ctx.layernorm_work(B.F16, -1, 4) == -1
    lib, h = ctx.lib, ctx.h
    st = torch.cuda.current_stream().cuda_stream
    p = x.data_ptr()
    for args in ((B.I8, p, c), (B.F16, p + 1, c), (B.F16, p, c - 1), (B.F16, None, c)):          # dtype, misaligned, pitch below the channels, null
        dt, ptr, ld = args
        want = B.ERR_UNSUPPORTED if dt == B.I8 else B.ERR_INVALID_ARG
        assert lib.emc2_layernorm(h, dt, ptr, ld, None, 0, g1.data_ptr(), g1.data_ptr(), 1e-5, None, n, c, None, 0, y.data_ptr(), c, st) == want
        assert lib.emc2_recurrence(h, dt, ptr, ld, p, c, off.data_ptr(), 1, n, c, 0, None, y.data_ptr(), c, None, work.data_ptr(), 1 << 22, st) == want
        assert lib.emc2_ffn(h, dt, 0, ptr, ld, packed.data_ptr(), None, 0, None, n, c, f, y.data_ptr(), c, st) == want
        assert lib.emc2_recurrence_step(h, dt, ptr, ld, p, c, x.data_ptr(), n, c, x.data_ptr(), y.data_ptr(), c, st) == want
    assert lib.emc2_layernorm(None, B.F16, p, c, None, 0, None, None, 0.0, None, n, c, None, 0, p, c, st) == B.ERR_INVALID_ARG
    assert lib.emc2_ffn_pack(h, B.F16, w[0].data_ptr(), w[1].data_ptr(), w[2].data_ptr(), c, f, packed.data_ptr() + 8, st) == B.ERR_INVALID_ARG
    ctx.status_sync()
