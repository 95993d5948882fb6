"""The selective operators' calls on another device than their context's: refused before anything is launched (one GPU is enough: the context is told that it
belongs to another)."""
import pytest
import torch

from paper_2507_04123_amd import binding as B

pytestmark = pytest.mark.gpu
N, C, M, TAPS = 5, 16, 4, 3


def _calls(ctx):
    def rows(w=C):
        return torch.zeros((N, w), device="cuda")

    def f(*shape):
        return torch.zeros(shape, device="cuda")

    off = torch.tensor([0, 2, N], dtype=torch.int32, device="cuda")
    work = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    x, y, dt, b, c = rows(), rows(), rows(), rows(M), rows(M)
    a, w = f(C, M), f(TAPS, C)
    return {
        "causal_conv": lambda: ctx.causal_conv(B.F32, x, w, off, y),
        "causal_conv_backward": lambda: ctx.causal_conv_backward(B.F32, x, w, off, dt, y, f(TAPS, C), work),
        "causal_conv_step": lambda: ctx.causal_conv_step(B.F32, x, w, f(N, TAPS - 1, C), f(N, TAPS - 1, C), y),
        "gated_residual": lambda: ctx.gated_residual(B.F32, x, dt, f(C), f(1), y, 1e-5),
        "gated_residual_backward": lambda: ctx.gated_residual_backward(B.F32, x, dt, f(C), f(1), 1e-5, rows(), y, rows(), f(C), f(1), work),
        "selective_scan": lambda: ctx.selective_scan(B.F32, x, dt, a, b, c, off, y, work),
        "selective_scan_backward": lambda: ctx.selective_scan_backward(B.F32, x, dt, a, b, c, off, rows(), y, rows(), f(C, M), rows(M), rows(M), work),
        "selective_scan_step": lambda: ctx.selective_scan_step(B.F32, x, dt, a, b, c, f(N, C, M), f(N, C, M), y),
    }


def test_another_device_is_refused():
    ctx = B.Context(1, 1, 1)
    for call in _calls(ctx).values():
        call()
    ctx.status_sync()
    ctx.device += 1
    try:
        for call in _calls(ctx).values():
            with pytest.raises(ValueError, match="device"):
                call()
    finally:
        ctx.device -= 1


@pytest.mark.parametrize("name", ["x", "w", "offsets", "y"])
def test_host_operands_are_refused(name):
    ctx = B.Context(1, 1, 1)
    t = {"x": torch.zeros((N, C), device="cuda"), "w": torch.zeros((TAPS, C), device="cuda"),
         "offsets": torch.tensor([0, N], dtype=torch.int32, device="cuda"), "y": torch.zeros((N, C), device="cuda")}
    t[name] = t[name].cpu()
    with pytest.raises(ValueError, match=name):
        ctx.causal_conv(B.F32, t["x"], t["w"], t["offsets"], t["y"])
