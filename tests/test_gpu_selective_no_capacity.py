"""The selective operators along sequences, called with buffers of no rows: states are handed on, weights' gradients are zeros, and offsets that claim rows are
reported."""
import pytest
import torch

from paper_2507_04123_amd import binding as B

from selective_helpers import DT, TYPES, draw, work

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _calls(ctx, dtype, off, c=20, m=5, taps=4):
    """name -> a call and its results"""
    k, t = off.numel() - 1, DT[dtype]

    def rows(w=c):
        return torch.empty((0, w), dtype=TD[dtype], device="cuda")

    def f(*shape):
        return torch.full(shape, 9.0, device="cuda")

    w, a, kept, h0 = draw(1, taps, c).cuda(), -torch.exp(draw(2, c, m)).cuda(), draw(3, k, taps - 1, c).cuda(), draw(4, k, c, m).cuda()
    out = {n: f(*s) for n, s in (("dw", (taps, c)), ("dbias", (c,)), ("kept", kept.shape), ("dkept", kept.shape), ("last", h0.shape), ("dh0", h0.shape),
                                 ("da", (c, m)), ("dskip", (c,)), ("ddt_bias", (c,)))}
    scan, one = (rows(), rows(), a, rows(m), rows(m), off), f(c)
    return {
        "causal_conv": (lambda: ctx.causal_conv(t, rows(), w, off, rows(), before=kept, last=out["kept"]), {"kept": kept}),
        "causal_conv_backward": (lambda: ctx.causal_conv_backward(t, rows(), w, off, rows(), rows(), out["dw"], work(ctx.causal_conv_work(t, 0, c, taps)),
                                                                  dbias=out["dbias"], before=kept, dlast=kept, dbefore=out["dkept"]),
                                 {"dw": 0 * w, "dbias": 0 * one, "dkept": kept}),
        "selective_scan": (lambda: ctx.selective_scan(t, *scan, rows(), work(ctx.selective_scan_work(t, 0, c, m)), h0=h0, last=out["last"]), {"last": h0}),
        "selective_scan_backward": (lambda: ctx.selective_scan_backward(t, *scan, rows(), rows(), rows(), out["da"], rows(m), rows(m),
                                                                        work(ctx.selective_scan_work(t, 0, c, m)), skip=one, dskip=out["dskip"], dt_bias=one,
                                                                        ddt_bias=out["ddt_bias"], h0=h0, dlast=h0, dh0=out["dh0"]),
                                    {"da": 0 * a, "dskip": 0 * one, "ddt_bias": 0 * one, "dh0": h0}),
    }, out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets", [[0, 0], [0, 0, 0, 0], [0, 5], [0, 3, 7]])
def test_no_capacity(dtype, offsets):
    ctx = B.Context(1, 1, 1)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    calls, out = _calls(ctx, dtype, off)
    for name, (call, want) in calls.items():
        call()
        if offsets[-1]:
            with pytest.raises(B.Emc2Error) as e:
                ctx.status_sync()
            assert e.value.status == B.ERR_CAPACITY, name
        else:
            ctx.status_sync()
        for k, v in want.items():
            assert torch.equal(out[k], v), (name, k)
    ctx.close()
