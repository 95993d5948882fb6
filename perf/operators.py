"""Performance cases of the sequence operators: layer norm, gated linear recurrence, gated feed-forward network.

`listed()` names the standing cases, `draw(rng)` gives further ones of the same ranges.  `prepare(case, seed)` builds what a program
holds before a call (seeded inputs on the GPU; with `own` also a context, packed weights, output and work buffers), `run(state)` is one
pass through an operator, in its plain form or, with `own`, through the library's entry points, `work(case)` the bytes and operations a
pass cannot do without, `exact(case, seed)` the same outputs from the definitions in 64 bits.

Operators (rows = the voxels of packed frames, one behind the other):
  norm        y = layer norm of x, or of x + residual with the sum kept; `train`: also the gradients of x and of both weights
  recurrence  h_t = a_t h_{t-1} + (1 - a_t) x_t along every frame, a = sigmoid(gate), from a given state; `train`: also the gradients
  step        the recurrence for one row per frame, states updated in place (serving a stream)
  ffn         y = (act(x Wg) * (x Wu)) Wd, plus a residual; `train`: weights laid out anew, output and all gradients
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

_TD = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_EPS = 1e-5


def listed():
    return [
        # the rows one sweep adds to a stream: a single short call, latency is everything
        {"name": "norm_few_rows_f16", "op": "norm", "rows": 37, "channels": 64, "dtype": "f16", "residual": False, "train": False},
        # all voxels of eight 64-beam frames, the residual stream added on the way: serving a batch
        {"name": "norm_residual_8_frames_f16", "op": "norm", "rows": 613217, "channels": 64, "dtype": "f16", "residual": True, "train": False},
        # a training batch of wide voxel rows
        {"name": "norm_train_bf16", "op": "norm", "rows": 240001, "channels": 128, "dtype": "bf16", "residual": False, "train": True},
        # fused LiDAR and image rows of a width that is no power of two, full precision
        {"name": "norm_train_ragged_f32", "op": "norm", "rows": 20011, "channels": 90, "dtype": "f32", "residual": False, "train": True},
        # one new row for each of eight streams: the serving form
        {"name": "step_8_streams_f16", "op": "step", "frames": 8, "channels": 128, "dtype": "f16"},
        # eight whole frames: long sequences, few of them
        {"name": "recurrence_8_frames_f16", "op": "recurrence", "rows": 613217, "frames": 8, "channels": 64, "dtype": "f16", "backwards": False,
         "train": False},
        # a training batch of three ragged frames, scanned from their ends
        {"name": "recurrence_train_bf16", "op": "recurrence", "rows": 200003, "frames": 3, "channels": 128, "dtype": "bf16", "backwards": True,
         "train": True},
        # many short sequences of very different lengths (the voxels of single objects), some empty, full precision
        {"name": "recurrence_many_short_f32", "op": "recurrence", "rows": 150001, "frames": 9001, "channels": 96, "dtype": "f32", "backwards": False,
         "train": False},
        # the rows one sweep adds to a stream
        {"name": "ffn_few_rows_f16", "op": "ffn", "rows": 24, "channels": 128, "hidden": 512, "dtype": "f16", "act": "silu", "residual": True,
         "train": False},
        # all voxels of a batch of dense frames: serving at full size
        {"name": "ffn_300k_rows_f16", "op": "ffn", "rows": 300000, "channels": 128, "hidden": 512, "dtype": "f16", "act": "silu", "residual": True,
         "train": False},
        # a training batch
        {"name": "ffn_train_bf16", "op": "ffn", "rows": 100003, "channels": 64, "hidden": 256, "dtype": "bf16", "act": "silu", "residual": False,
         "train": True},
        # a training batch in full precision, odd widths
        {"name": "ffn_train_ragged_f32", "op": "ffn", "rows": 7001, "channels": 48, "hidden": 200, "dtype": "f32", "act": "gelu", "residual": False,
         "train": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Channels: half the time a multiple of 16, else anything."""
    c = _log_int(rng, lo, hi)
    return max(16, c // 16 * 16) if rng.random() < 0.5 else c


def draw(rng):
    op = rng.choice(["norm", "norm", "recurrence", "recurrence", "step", "ffn", "ffn", "ffn"])
    dtype = rng.choice(["f16", "bf16", "f32"])
    train = rng.random() < 0.5
    if op == "norm":
        channels = _width(rng, 8, 1024)
        return {"op": op, "rows": min(_log_int(rng, 1, 600000), 16000000 // channels), "channels": channels, "dtype": dtype,
                "residual": not train and rng.random() < 0.5, "train": train}
    if op == "step":
        return {"op": op, "frames": _log_int(rng, 1, 4096), "channels": _width(rng, 8, 512), "dtype": dtype}
    if op == "recurrence":
        channels = _width(rng, 8, 512)
        rows = min(_log_int(rng, 1, 600000), 16000000 // channels)
        return {"op": op, "rows": rows, "frames": _log_int(rng, 1, max(1, rows // 8)), "channels": channels, "dtype": dtype,
                "backwards": rng.random() < 0.5, "train": train}
    channels, hidden = _width(rng, 8, 256), _width(rng, 16, 1024)
    room = 2000000000 // (channels * hidden) if dtype == "f32" or train else 16000000000 // (channels * hidden)
    return {"op": op, "rows": min(_log_int(rng, 1, 300000), room), "channels": channels, "hidden": hidden, "dtype": dtype,
            "act": rng.choice(["silu", "gelu"]), "residual": not train and rng.random() < 0.5, "train": train}


# --------------------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------------------

def _offsets(rows, frames, seed):
    """First rows of the sequences, [frames + 1]: lengths of a wide spread that add up to `rows`, one in nine of many empty."""
    r = np.random.RandomState(seed % (1 << 31))
    share = r.exponential(size=frames) + 0.02
    if frames >= 9:
        share[r.permutation(frames)[: frames // 9]] = 0.0
    ends = np.floor(np.cumsum(share) / share.sum() * rows + 0.5).astype(np.int64)
    ends[-1] = rows
    return np.concatenate([[0], np.minimum(ends, rows)])


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    td, c = _TD[case["dtype"]], case["channels"]

    def randn(*shape, scale=1.0, shift=0.0, to=td):
        return (torch.randn(shape, generator=g, device="cuda") * scale + shift).to(to)

    n = case["rows"] if case["op"] != "step" else case["frames"]
    s = {"x": randn(n, c)}
    if case["op"] == "norm":
        # rows of different magnitude with a common offset, as behind a ReLU; every 64th a row of zeros (a voxel without a match)
        scale = torch.exp(torch.randn((n, 1), generator=g, device="cuda"))
        s["x"] = (s["x"].float() * scale + 0.5 * scale).to(td)
        s["x"][5::64] = 0
        s["gamma"], s["beta"] = randn(c, scale=0.2, shift=1.0, to=torch.float32), randn(c, scale=0.2, to=torch.float32)
        if case["residual"]:
            s["residual"] = randn(n, c)
        if case["train"]:
            s["dy"] = randn(n, c)
    elif case["op"] in ("recurrence", "step"):
        # gates mostly open (a long memory), a few shut hard
        s["gate"] = randn(n, c, scale=2.0, shift=2.0)
        s["gate"][::37] = randn(*s["gate"][::37].shape, scale=20.0)
        s["h0"] = randn(case["frames"], c, to=torch.float32)
        if case["op"] == "recurrence":
            off = _offsets(n, case["frames"], seed)
            s["longest"] = int(np.max(np.diff(off)))
            s["offsets"] = torch.from_numpy(off.astype(np.int32)).cuda()
            if case["train"]:
                s["dy"], s["dlast"] = randn(n, c), randn(case["frames"], c, to=torch.float32)
    else:
        f = case["hidden"]
        s["wg"], s["wu"] = randn(c, f, scale=c ** -0.5), randn(c, f, scale=c ** -0.5)
        s["wd"] = randn(f, c, scale=f ** -0.5)
        if case["residual"]:
            s["residual"] = randn(n, c)
        if case["train"]:
            s["dy"] = randn(n, c)
    return s


@functools.lru_cache(maxsize=None)
def _context():
    from paper_2507_04123_amd import binding as B
    return B.Context(1, 1, 1)


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    return {**s, **_held(case, s)} if own else s


def _held(case, s):
    """What a program that calls the library keeps beside its inputs: the context, packed weights, buffers."""
    from paper_2507_04123_amd import binding as B
    ctx, c, n = _context(), case["channels"], s["x"].shape[0]
    dt = {"f32": B.F32, "f16": B.F16, "bf16": B.BF16}[case["dtype"]]
    new = {"ctx": ctx, "dt": dt, "y": torch.empty_like(s["x"])}

    def work(size):
        return torch.empty(size, dtype=torch.uint8, device="cuda")

    if case["op"] == "norm":
        if case["residual"]:
            new["sum"] = torch.empty_like(s["x"])
        if case["train"]:
            new.update(dx=torch.empty_like(s["x"]), dgamma=torch.empty_like(s["gamma"]), dbeta=torch.empty_like(s["gamma"]),
                       work=work(ctx.layernorm_work(dt, n, c)))
    elif case["op"] == "recurrence":
        new.update(last=torch.empty_like(s["h0"]), work=work(ctx.recurrence_work(dt, n, c)))
        if case["train"]:
            new.update(dx=torch.empty_like(s["x"]), dgate=torch.empty_like(s["x"]), dh0=torch.empty_like(s["h0"]))
    elif case["op"] == "step":
        new["h"] = s["h0"].clone()
    else:
        f = case["hidden"]
        new["act"] = {"silu": B.ACT_SILU, "gelu": B.ACT_GELU}[case["act"]]
        new["packed"] = torch.empty(ctx.ffn_packed_size(dt, c, f), dtype=_TD[case["dtype"]], device="cuda")
        if case["train"]:
            new.update(dx=torch.empty_like(s["x"]), dwg=torch.empty_like(s["wg"]), dwu=torch.empty_like(s["wu"]), dwd=torch.empty_like(s["wd"]),
                       work=work(ctx.ffn_work(dt, n, c, f)))
        else:
            ctx.ffn_pack(dt, s["wg"], s["wu"], s["wd"], new["packed"])
    return new


# --------------------------------------------------------------------------------------------------------------
# run
# --------------------------------------------------------------------------------------------------------------

def run(state):
    return _RUN[state["case"]["op"], own](state)


def _norm_own(s):
    s["ctx"].layernorm(s["dt"], s["x"], s["gamma"], s["beta"], _EPS, s["y"], residual=s.get("residual"), total=s.get("sum"))
    if not s["case"]["train"]:
        return {k: s[k] for k in ("y", "sum") if k in s}
    s["ctx"].layernorm_backward(s["dt"], s["x"], s["gamma"], _EPS, s["dy"], s["dx"], s["dgamma"], s["dbeta"], s["work"])
    return {k: s[k] for k in ("y", "dx", "dgamma", "dbeta")}


def _norm_plain(s):
    x, td = s["x"].float(), s["x"].dtype
    out = {}
    if "residual" in s:
        x = x + s["residual"].float()
        out["sum"] = x.to(td)
    d = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + _EPS)
    xh = d * rstd
    out["y"] = (xh * s["gamma"] + s["beta"]).to(td)
    if "dy" in s:
        dy = s["dy"].float()
        gy = dy * s["gamma"]
        out["dx"] = (rstd * (gy - gy.mean(1, keepdim=True) - xh * (gy * xh).mean(1, keepdim=True))).to(td)
        out["dgamma"], out["dbeta"] = (dy * xh).sum(0), dy.sum(0)
    return out


def _recurrence_own(s):
    back = s["case"]["backwards"]
    s["ctx"].recurrence(s["dt"], s["x"], s["gate"], s["offsets"], s["y"], s["work"], backwards=back, h0=s["h0"], last=s["last"])
    if not s["case"]["train"]:
        return {k: s[k] for k in ("y", "last")}
    s["ctx"].recurrence_backward(s["dt"], s["x"], s["gate"], s["offsets"], s["dy"], s["dx"], s["dgate"], s["work"], backwards=back, h0=s["h0"],
                                 dlast=s["dlast"], dh0=s["dh0"])
    return {k: s[k] for k in ("y", "last", "dx", "dgate", "dh0")}


def _scan(a, b, longest):
    """u_t = a_t u_{t-1} + b_t by doubling; a_t = 0 where a sequence of at most `longest` rows begins."""
    step = 1
    while step < longest:
        b = torch.cat([b[:step], b[step:] + a[step:] * b[:-step]])
        a = torch.cat([a[:step], a[step:] * a[:-step]])
        step *= 2
    return b


def _recurrence_plain(s):
    td, n, back = s["x"].dtype, s["x"].shape[0], s["case"]["backwards"]
    x, gate, off = s["x"].float(), s["gate"].float(), s["offsets"].long()
    first, last = off[:-1], off[1:] - 1                       # of every sequence, in the order of the rows
    if back:
        x, gate = x.flip(0), gate.flip(0)
        first, last = n - 1 - last, n - 1 - first
    some = last >= first
    at_first, at_last = first[some], last[some]
    keep, take = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
    a, b = keep.clone(), take * x
    b[at_first] += keep[at_first] * s["h0"][some]
    a[at_first] = 0
    h = _scan(a, b, s["longest"])
    out_last = s["h0"].clone()
    out_last[some] = h[at_last]
    turn = (lambda t: t.flip(0)) if back else (lambda t: t)
    out = {"y": turn(h).to(td), "last": out_last}
    if "dy" in s:
        dy = turn(s["dy"].float()).clone()
        dy[at_last] += s["dlast"][some]
        nxt = torch.zeros_like(keep)                          # the gate of the row behind, none behind a sequence's last
        nxt[:-1] = keep[1:]
        nxt[at_last] = 0
        du = _scan(nxt.flip(0), dy.flip(0), s["longest"]).flip(0)
        prev = torch.zeros_like(h)
        prev[1:] = h[:-1]
        prev[at_first] = s["h0"][some]
        dh0 = s["dlast"].clone()
        dh0[some] = keep[at_first] * du[at_first]
        out.update(dx=turn(take * du).to(td), dgate=turn(du * (prev - x) * keep * take).to(td), dh0=dh0)
    return out


def _step_own(s):
    s["ctx"].recurrence_step(s["dt"], s["x"], s["gate"], s["h0"], s["h"], s["y"])
    return {k: s[k] for k in ("y", "h")}


def _step_plain(s):
    x, gate = s["x"].float(), s["gate"].float()
    h = s["h0"] / (1 + torch.exp(-gate)) + x / (1 + torch.exp(gate))
    return {"y": h.to(s["x"].dtype), "h": h}


def _ffn_own(s):
    ctx, f = s["ctx"], s["case"]["hidden"]
    if s["case"]["train"]:
        ctx.ffn_pack(s["dt"], s["wg"], s["wu"], s["wd"], s["packed"])
    ctx.ffn(s["dt"], s["act"], s["x"], s["packed"], f, s["y"], residual=s.get("residual"))
    if not s["case"]["train"]:
        return {"y": s["y"]}
    ctx.ffn_backward(s["dt"], s["act"], s["x"], s["packed"], f, s["dy"], s["dx"], s["dwg"], s["dwu"], s["dwd"], s["work"])
    return {k: s[k] for k in ("y", "dx", "dwg", "dwu", "dwd")}


_GELU = math.sqrt(2 / math.pi)


def _ffn_plain(s):
    td, x = s["x"].dtype, s["x"].float()
    wg, wu, wd = s["wg"].float(), s["wu"].float(), s["wd"].float()
    gate, up = x @ wg, x @ wu
    if s["case"]["act"] == "silu":
        on = 1 / (1 + torch.exp(-gate))
        act, slope = gate * on, on * (1 + gate * (1 - on))
    else:
        t = torch.tanh(_GELU * (gate + 0.044715 * gate ** 3))
        act, slope = 0.5 * gate * (1 + t), 0.5 * (1 + t) + 0.5 * gate * (1 - t * t) * _GELU * (1 + 3 * 0.044715 * gate * gate)
    hid = act * up
    y = hid @ wd
    if "residual" in s:
        y = y + s["residual"].float()
    out = {"y": y.to(td)}
    if "dy" in s:
        dy = s["dy"].float()
        dh = dy @ wd.t()
        dgate, dup = dh * up * slope, dh * act
        out.update(dx=(dgate @ wg.t() + dup @ wu.t()).to(td), dwg=(x.t() @ dgate).to(td), dwu=(x.t() @ dup).to(td), dwd=(hid.t() @ dy).to(td))
    return out


_RUN = {("norm", True): _norm_own, ("norm", False): _norm_plain, ("recurrence", True): _recurrence_own, ("recurrence", False): _recurrence_plain,
        ("step", True): _step_own, ("step", False): _step_plain, ("ffn", True): _ffn_own, ("ffn", False): _ffn_plain}


# --------------------------------------------------------------------------------------------------------------
# work, exact
# --------------------------------------------------------------------------------------------------------------

def work(case):
    size, c, train = _BYTES[case["dtype"]], case["channels"], case.get("train", False)
    if case["op"] == "step":
        n = case["frames"]
        return {"bytes": n * c * (3 * size + 8), "flops": 6 * n * c}
    n = case["rows"]
    if case["op"] == "norm":
        rows = 4 if train or case["residual"] else 2          # x, y and dy, dx or residual, sum
        return {"bytes": rows * n * c * size + (16 if train else 8) * c, "flops": (24 if train else 8) * n * c}
    if case["op"] == "recurrence":
        rows, states = (6, 4) if train else (3, 2)            # x, gate, y and dy, dx, dgate
        return {"bytes": rows * n * c * size + states * case["frames"] * c * 4 + 4 * case["frames"], "flops": (24 if train else 8) * n * c}
    f = case["hidden"]
    rows = 4 if train else 2 + bool(case["residual"])
    products = 9 if train else 3                              # with the gradients: dH, two of dx, three of the weights
    return {"bytes": rows * n * c * size + (6 if train else 3) * c * f * size, "flops": 2 * products * n * c * f}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] in ("recurrence", "step"):
        return _recurrence_exact(case, s)
    v = {k: t.double() for k, t in s.items()}
    wanted = {"norm": ("x", "gamma", "beta"), "ffn": ("x", "wg", "wu", "wd")}[case["op"]]
    for k in wanted:
        v[k].requires_grad_(case["train"])
    if case["op"] == "norm":
        x = v["x"] + v["residual"] if case["residual"] else v["x"]
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        y = (x - mean) / torch.sqrt(var + _EPS) * v["gamma"] + v["beta"]
    else:
        z = v["x"] @ v["wg"]
        z = z * torch.sigmoid(z) if case["act"] == "silu" else torch.nn.functional.gelu(z, approximate="tanh")
        y = (z * (v["x"] @ v["wu"])) @ v["wd"]
        if case["residual"]:
            y = y + v["residual"]
    out = {"y": y.detach()}
    if case["op"] == "norm" and case["residual"]:
        out["sum"] = x.detach()
    if case["train"]:
        y.backward(v["dy"])
        out.update({"d" + k: v[k].grad for k in wanted})
    return out


def _recurrence_exact(case, s):
    """Row after row, as the definition says."""
    x, gate, h0 = (s[k].double().cpu().numpy() for k in ("x", "gate", "h0"))
    keep, take = 1 / (1 + np.exp(-gate)), 1 / (1 + np.exp(gate))
    if case["op"] == "step":
        h = keep * h0 + take * x
        return {"y": h, "h": h}
    off = s["offsets"].cpu().numpy()
    new = take * x
    y, last = np.empty_like(x), h0.copy()
    for i in range(case["frames"]):
        order = range(off[i], off[i + 1])
        h = h0[i]
        for t in (reversed(order) if case["backwards"] else order):
            h = keep[t] * h + new[t]
            y[t] = h
        last[i] = h
    out = {"y": y, "last": last}
    if case["train"]:
        dy, flow = s["dy"].double().cpu().numpy(), s["dlast"].double().cpu().numpy()
        du = np.empty_like(x)
        prev = np.empty_like(x)
        for i in range(case["frames"]):
            lo, hi = off[i], off[i + 1]
            if lo == hi:
                continue
            if case["backwards"]:
                prev[hi - 1], prev[lo:hi - 1], order = h0[i], y[lo + 1:hi], range(lo, hi)
            else:
                prev[lo], prev[lo + 1:hi], order = h0[i], y[lo:hi - 1], reversed(range(lo, hi))
            d = flow[i]
            for t in order:
                du[t] = dy[t] + d
                d = keep[t] * du[t]
            flow[i] = d
        out.update(dx=take * du, dgate=du * (prev - x) * keep * take, dh0=flow)
    return out
