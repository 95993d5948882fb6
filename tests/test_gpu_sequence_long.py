"""The sequence operators at sizes where a wave or block walks several tiles of rows and the parts of a sum are many, against the oracle in 64
bits within the bounds that the number formats give.  Wide rows reach such sizes with few of them: a recurrence's blocks, 512 in all, are shared out over
the slices of 64 (fp32: 32) channels."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from paper_2507_04123_amd import binding as B

import sequence_bounds as L

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DT = {"f32": B.F32, "f16": B.F16, "bf16": B.BF16}


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


def _normal(seed, *shape, scale=1.0, shift=0.0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale + shift).to(dtype)


def _np(t):
    return t.double().cpu().numpy()


def _within(got, exp, bound, what):
    got = _np(got)
    bad = ~(np.abs(got - exp) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside, first {i}: {got[i]!r}, {exp[i]!r} +- {bound[i]:.3g}")


def _work(size):
    return torch.full((max(size, 16),), 0xA5, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------------------ recurrence

def _offsets(kind, n):
    """One sequence; or starts and ends at and beside multiples of 16 to 4096 rows, some twice (an empty sequence), with long stretches between."""
    if kind == "one":
        return np.array([0, n])
    r = np.random.RandomState(n)
    at = [m * k + d for m in (16, 64, 128, 256, 1024, 2048, 4096) for k in r.randint(1, max(2, n // m), 3) for d in (-1, 0, 1)]
    at = sorted(a for a in at if 0 < a < n // 3 or 2 * n // 3 < a < n)
    return np.sort(np.array([0, 0] + at + at[::5] + [n, n]))


def _recurrence(ctx, dtype, c, n, off, backwards, spare, compare):
    """Both passes over n rows (of n + spare in the buffers, the others NaN); `compare` gets the operands and results of the rows present."""
    td, dt = TD[dtype], DT[dtype]
    cap, seqs = n + spare, len(off) - 1
    x, gate, dy = _normal(1, cap, c, dtype=td), _normal(2, cap, c, scale=2.0, shift=2.5, dtype=td), _normal(3, cap, c, dtype=td)
    for t in (x, gate, dy):
        t[n:] = float("nan")
    h0, dlast, offsets = _normal(4, seqs, c), _normal(5, seqs, c), torch.from_numpy(off.astype(np.int32)).cuda()
    y, dx, dgate = (torch.full_like(x, 7.0) for _ in range(3))
    last, dh0 = torch.full_like(h0, 7.0), torch.full_like(h0, 7.0)
    work = _work(ctx.recurrence_work(dt, cap, c))
    ctx.recurrence(dt, x, gate, offsets, y, work, backwards=backwards, h0=h0, last=last)
    ctx.recurrence_backward(dt, x, gate, offsets, dy, dx, dgate, work, backwards=backwards, h0=h0, dlast=dlast, dh0=dh0)
    ctx.status_sync()
    assert all(bool((t[n:] == 7.0).all()) for t in (y, dx, dgate))
    compare([x[:n], gate[:n], h0, dy[:n], dlast], [y[:n], last, dx[:n], dgate[:n], dh0])


# f16 and bf16: 24 tiles of 128 rows (gradients: 47 of 64) in blocks of 2 (3); 64 in 8 blocks of 8 (128 in 8 of 16); 71 in 3 blocks of 32 at most (141 in 5).
# fp32: 20 tiles of 256 (40 of 128) in blocks of 3 (5); 36 in 2 blocks of 32 at most (71 in 3); as many channels as there may be in one block
@pytest.mark.parametrize("dtype,c,n", [("f16", 2048, 3000), ("bf16", 4096, 8190), ("f16", 16384, 9000), ("f32", 2047, 5001), ("f32", 16384, 9001),
                                       ("f16", 65536, 300), ("f32", 65533, 700)])
@pytest.mark.parametrize("kind", ["one", "edges"])
@pytest.mark.parametrize("backwards", [False, True])
def test_recurrence_over_several_tiles(ctx, dtype, c, n, kind, backwards):
    off = _offsets(kind, n)
    r = np.random.RandomState(c)
    cols = sorted({0, 1, 63, 64, c - 65, c - 4, c - 1, *r.randint(0, c, 17)})         # channels do not meet: a few of them are compared

    def compare(operands, results):
        x, gate, h0, dy, dlast = (_np(t[:, cols]) for t in operands)
        y, last = S.recurrence(x, gate, off, h0, backwards)
        by, bl, _ = L.recurrence(x, gate, off, h0, backwards, dtype)
        exp = (y, last, *S.recurrence_backward(x, gate, off, h0, dy, dlast, backwards))
        bounds = (by, bl, *L.recurrence_backward(x, gate, off, h0, dy, dlast, backwards, dtype))
        for got, e, b, what in zip(results, exp, bounds, ("y", "last", "dx", "dgate", "dh0")):
            _within(got[:, cols], e, b, what)

    _recurrence(ctx, dtype, c, n, off, backwards, 700 if kind == "edges" else 0, compare)


# rows of 1 to 64 channels need many: 2 to 4 tiles a block of 512.  Sequences of one length, which the oracle takes as channels of one
@pytest.mark.parametrize("dtype,c,length,seqs", [("f32", 1, 1000, 2200), ("f16", 3, 2500, 400), ("bf16", 7, 777, 700), ("f16", 64, 10000, 14), ("f32", 33, 1, 70000)])
@pytest.mark.parametrize("backwards", [False, True])
def test_recurrence_of_narrow_rows_over_several_tiles(ctx, dtype, c, length, seqs, backwards):
    off, one = np.arange(seqs + 1) * length, np.array([0, length])

    def compare(operands, results):
        def rows(t):
            return _np(t).reshape(seqs, length, c).transpose(1, 0, 2).reshape(length, seqs * c)

        def states(t):
            return _np(t).reshape(1, seqs * c)

        x, gate, dy, h0, dlast = rows(operands[0]), rows(operands[1]), rows(operands[3]), states(operands[2]), states(operands[4])
        y, last = S.recurrence(x, gate, one, h0, backwards)
        by, bl, _ = L.recurrence(x, gate, one, h0, backwards, dtype)
        exp = (y, last, *S.recurrence_backward(x, gate, one, h0, dy, dlast, backwards))
        bounds = (by, bl, *L.recurrence_backward(x, gate, one, h0, dy, dlast, backwards, dtype))
        for got, e, b, what in zip(results, exp, bounds, ("y", "last", "dx", "dgate", "dh0")):
            form = rows if what in ("y", "dx", "dgate") else states
            _within(torch.from_numpy(form(got)), e, b, what)

    _recurrence(ctx, dtype, c, seqs * length, off, backwards, 99, compare)


# ------------------------------------------------------------------------------------------------------------ layer norm

# blocks: 1280 (several vectors a lane: 768), each walking two to five times; 1250 walking once; 257
@pytest.mark.parametrize("dtype,c,n", [("f32", 5, 200001), ("f16", 20, 300000), ("bf16", 90, 60001), ("f16", 1000, 9001), ("f32", 1024, 7000), ("f32", 90, 20000),
                                       ("f16", 64, 16448)])
def test_layernorm_backward_of_many_blocks(ctx, dtype, c, n):
    td = TD[dtype]
    x, dy, add, gamma = _normal(1, n, c, scale=2.0, shift=1.0, dtype=td), _normal(2, n, c, dtype=td), _normal(3, n, c, dtype=td), _normal(4, c, scale=0.3, shift=1.0)
    x[::64] = 0
    dx, dg, db = torch.full_like(x, 7.0), torch.full_like(gamma, 7.0), torch.full_like(gamma, 7.0)
    ctx.layernorm_backward(DT[dtype], x, gamma, 1e-5, dy, dx, dg, db, _work(ctx.layernorm_work(DT[dtype], n, c)), add=add)
    xs, g, d, ad = _np(x), _np(gamma), _np(dy), _np(add)
    ex, eg, eb = S.layernorm_backward(xs, g, 1e-5, d)
    bx, bg, bb = L.layernorm_backward(xs, g, 1e-5, d, ad, dtype)
    _within(dx, ex + ad, bx, "dx")
    _within(dg, eg, bg, "dgamma")
    _within(db, eb, bb, "dbeta")


# ------------------------------------------------------------------------------------------------------------ feed-forward

def _network(ctx, dtype, c, f):
    w = [_normal(10 + i, *s, scale=s[0] ** -0.5, dtype=TD[dtype]) for i, s in enumerate(((c, f), (c, f), (f, c)))]
    packed = torch.full((ctx.ffn_packed_size(DT[dtype], c, f),), float("nan"), dtype=TD[dtype], device="cuda")
    ctx.ffn_pack(DT[dtype], *w, packed)
    return w, [_np(t) for t in w], packed


@pytest.mark.parametrize("dtype,c", [("f16", 64), ("bf16", 40), ("f16", 160), ("f32", 32), ("f32", 90), ("f32", 160)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_ffn_many_rows_in_place_with_a_device_count(ctx, dtype, c, act):
    """40 000 rows: waves with rows of their own; NaN in the rows beyond the count; results where operands lie."""
    f, cap, dt, code = 72, 40000, DT[dtype], B.ACT_SILU if act == "silu" else B.ACT_GELU
    w, ws, packed = _network(ctx, dtype, c, f)
    x, dy = _normal(1, cap, c, dtype=TD[dtype]), _normal(2, cap, c, dtype=TD[dtype])
    work = _work(ctx.ffn_work(dt, cap, c, f))
    for n in (0, 1, 20001, cap):
        count = torch.tensor([n], dtype=torch.int32, device="cuda")
        poison, flow, y = x.clone(), dy.clone(), x.clone()
        for t in (poison, flow, y):
            t[n:] = float("nan")
        ctx.ffn(dt, code, y, packed, f, y, residual=y, n=count)                        # residual, operand and result in one place
        g = [torch.full_like(t, 9.0) for t in w]
        ctx.ffn_backward(dt, code, poison, packed, f, flow, flow, *g, work, n=count)   # dx where dy lies
        where = poison.clone()
        ctx.ffn_backward(dt, code, where, packed, f, torch.where(torch.isnan(poison), poison, dy), where, *[torch.empty_like(t) for t in w], work, n=count)   # and where x does
        assert all(bool(torch.isnan(t[n:]).all()) for t in (y, flow, where)) and torch.equal(where[:n], flow[:n])
        if n == 0:
            assert not any(t.any() for t in g)
            continue
        xs, ds = _np(x[:n]), _np(dy[:n])
        _within(y[:n], S.ffn(act, xs, *ws) + xs, L.ffn(act, xs, *ws, xs, dtype), f"y {n}")
        for got, e, b, what in zip((flow[:n], *g), S.ffn_backward(act, xs, *ws, ds), L.ffn_backward(act, xs, *ws, ds, dtype), ("dx", "dwg", "dwu", "dwd")):
            _within(got, e, b, f"{what} {n}")


@pytest.mark.parametrize("dtype,c,f,rows", [("f16", 96, 30001, 300), ("f32", 40, 50001, 130), ("bf16", 16, 65536, 300), ("bf16", 250, 24600, 40)])
def test_ffn_of_more_slices_than_the_chip_holds_blocks(ctx, dtype, c, f, rows):
    w, ws, packed = _network(ctx, dtype, c, f)
    x, dy = _normal(1, rows, c, dtype=TD[dtype]), _normal(2, rows, c, dtype=TD[dtype])
    y, dx, g = torch.full_like(x, 7.0), torch.full_like(x, 7.0), [torch.full_like(t, 9.0) for t in w]
    ctx.ffn(DT[dtype], B.ACT_SILU, x, packed, f, y)
    ctx.ffn_backward(DT[dtype], B.ACT_SILU, x, packed, f, dy, dx, *g, _work(ctx.ffn_work(DT[dtype], rows, c, f)))
    xs, ds = _np(x), _np(dy)
    _within(y, S.ffn("silu", xs, *ws), L.ffn("silu", xs, *ws, np.zeros_like(xs), dtype), "y")
    for got, e, b, what in zip((dx, *g), S.ffn_backward("silu", xs, *ws, ds), L.ffn_backward("silu", xs, *ws, ds, dtype), ("dx", "dwg", "dwu", "dwd")):
        _within(got, e, b, what)
