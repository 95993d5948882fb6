"""A block over the voxels of packed frames: layer norm, gated feed-forward network, gated linear recurrence; run, trained and served.

    u = layernorm(x),  v = x + ffn(u),  gate = layernorm'(x),  y = recurrence(v, gate) along every frame's voxels

A 3x3x3 convolution sees 27 cells; the recurrence carries a state along a frame's whole voxel list (ascending key), from its first voxel to
its last or backwards.  As in ``pipeline``, only call order and buffers live here: everything is allocated once, ``run``, ``backward`` and
``step`` allocate nothing and never wait for the GPU, and counts stay in device memory.
"""
from __future__ import annotations

from typing import Dict, Optional

import torch

from . import binding as B
from .configs import F32, F16, BF16

_TD = {F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16}
_EPS = 1e-5


def sequence_params(params: Dict, dtype: int, device: str = "cuda") -> Dict[str, torch.Tensor]:
    """Host parameters (gen.make_sequence_params) on the device: weights in `dtype`, the layer norms' in fp32."""
    return {k: torch.from_numpy(v).to(device).to(_TD[dtype] if k[0] == "w" else torch.float32).contiguous() for k, v in params.items()}


class SequenceBlock:
    """One block over up to `capacity` rows in `n_frames` frames.  `train`: also holds what backward() needs."""

    def __init__(self, ctx: B.Context, dtype: int, capacity: int, n_frames: int, params: Dict[str, torch.Tensor],
                 activation: int = B.ACT_SILU, backwards: bool = False, train: bool = False, device: str = "cuda"):
        self.ctx, self.dtype, self.activation, self.backwards = ctx, dtype, activation, backwards
        self.channels, self.hidden = (int(v) for v in params["wg"].shape)
        c, td = self.channels, _TD[dtype]

        def rows():
            return torch.empty((capacity, c), dtype=td, device=device)

        self.u, self.v, self.gate, self.y = rows(), rows(), rows(), rows()
        self.offsets = torch.zeros(n_frames + 1, dtype=torch.int32, device=device)
        self.last = torch.zeros((n_frames, c), dtype=torch.float32, device=device)
        self.packed = torch.empty(ctx.ffn_packed_size(dtype, c, self.hidden), dtype=td, device=device)
        need = ctx.recurrence_work(dtype, capacity, c)
        self.grads: Optional[Dict[str, torch.Tensor]] = None
        if train:
            need = max(need, ctx.layernorm_work(dtype, capacity, c), ctx.ffn_work(dtype, capacity, c, self.hidden))
            self.dv, self.dgate, self.du, self.dx = rows(), rows(), rows(), rows()
            self.dh0 = torch.zeros_like(self.last)
            self.grads = {k: torch.zeros_like(t) for k, t in params.items()}
        self.work = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
        self.load(params)

    def load(self, params: Dict[str, torch.Tensor]) -> None:
        """Takes the parameters over: the tensors are kept, the weights' fragments made of them.  Call it again when they have changed."""
        c, f = self.channels, self.hidden
        shapes = {"wg": (c, f), "wu": (c, f), "wd": (f, c), "gamma": (c,), "beta": (c,), "gate_gamma": (c,), "gate_beta": (c,)}
        got = {k: tuple(params[k].shape) if k in params else None for k in shapes}
        if got != shapes:
            raise ValueError(f"load: need parameters of {shapes}, got {got}")
        self.ctx.ffn_pack(self.dtype, params["wg"], params["wu"], params["wd"], self.packed)
        self.params = params

    def find_frames(self, coords: torch.Tensor, n: torch.Tensor, capacity: int) -> torch.Tensor:
        """First row of every frame of a voxel list (its coordinates and device count), into self.offsets."""
        self.ctx.frame_offsets(coords, n, capacity, self.offsets.numel() - 1, self.offsets)
        return self.offsets

    def run(self, x: torch.Tensor, offsets: torch.Tensor, h0: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [rows][channels] of packed frames -> y of as many rows; the states behind each frame's last voxel go to self.last (of which h0, to go
        on from there, has to be a copy)."""
        ctx, p, n, k = self.ctx, self.params, offsets[-1:], x.shape[0]
        u, v, gate, y = self.u[:k], self.v[:k], self.gate[:k], self.y[:k]
        ctx.layernorm(self.dtype, x, p["gamma"], p["beta"], _EPS, u, n=n)
        ctx.ffn(self.dtype, self.activation, u, self.packed, self.hidden, v, residual=x, n=n)
        ctx.layernorm(self.dtype, x, p["gate_gamma"], p["gate_beta"], _EPS, gate, n=n)
        ctx.recurrence(self.dtype, v, gate, offsets, y, self.work, backwards=self.backwards, h0=h0, last=self.last)
        return y

    def backward(self, x: torch.Tensor, offsets: torch.Tensor, dy: torch.Tensor, h0: Optional[torch.Tensor] = None,
                 dlast: Optional[torch.Tensor] = None) -> torch.Tensor:
        """dx of the last run() over the same rows; the parameters' gradients go to self.grads, that of h0 to self.dh0."""
        if self.grads is None:
            raise ValueError("backward: the block was made without train=True")
        ctx, p, g, n, k = self.ctx, self.params, self.grads, offsets[-1:], x.shape[0]
        u, v, gate = self.u[:k], self.v[:k], self.gate[:k]
        dv, dgate, du, dx = self.dv[:k], self.dgate[:k], self.du[:k], self.dx[:k]
        ctx.recurrence_backward(self.dtype, v, gate, offsets, dy, dv, dgate, self.work, backwards=self.backwards, h0=h0, dlast=dlast,
                                dh0=self.dh0)
        ctx.ffn_backward(self.dtype, self.activation, u, self.packed, self.hidden, dv, du, g["wg"], g["wu"], g["wd"], self.work, n=n)
        ctx.layernorm_backward(self.dtype, x, p["gamma"], _EPS, du, dx, g["gamma"], g["beta"], self.work, add=dv, n=n)
        ctx.layernorm_backward(self.dtype, x, p["gate_gamma"], _EPS, dgate, dx, g["gate_gamma"], g["gate_beta"], self.work, add=dx, n=n)
        return dx

    def step(self, x: torch.Tensor, h: torch.Tensor) -> torch.Tensor:
        """One new row per frame, x [frames][channels]: the frames' states h (fp32) move on in place; returns y (where run()'s lies).  What a
        backward() still to come reads of the last run() is left as it is: a training block's step works in that pass's own buffers."""
        ctx, p, k = self.ctx, self.params, x.shape[0]
        u, v, gate = (self.u, self.v, self.gate) if self.grads is None else (self.du, self.dv, self.dgate)
        u, v, gate, y = u[:k], v[:k], gate[:k], self.y[:k]
        ctx.layernorm(self.dtype, x, p["gamma"], p["beta"], _EPS, u)
        ctx.ffn(self.dtype, self.activation, u, self.packed, self.hidden, v, residual=x)
        ctx.layernorm(self.dtype, x, p["gate_gamma"], p["gate_beta"], _EPS, gate)
        ctx.recurrence_step(self.dtype, v, gate, h, h, y)
        return y
