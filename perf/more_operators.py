"""Performance cases of the selective state space operators: short causal convolution, selective scan, gated residual with its norms.

`listed()` names the standing cases, `draw(rng)` gives further ones of the same ranges.  `prepare(case, seed)` builds what a program
holds before a call (seeded inputs on the GPU; with `own` also a context, output and work buffers), `run(state)` is one pass through an
operator, in its plain form or, with `own`, through the library's entry points, `work(case)` the bytes and operations a pass cannot do
without, `exact(case, seed)` the same outputs from the definitions in 64 bits.

Operators (rows = the voxels of packed frames, one behind the other):
  conv        y_t = silu(bias + sum_k w[k] x_{t-k}) along every frame, rows before the first given; `train`: also the gradients
  conv_step   the convolution for one row per frame, the rows kept of each frame moving on (serving a stream)
  scan        h_t = exp(D_t A) h_{t-1} + D_t x_t B_t,  y_t = C_t . h_t + skip x_t along every frame, D = softplus(dt + bias); `train`: also
              the gradients
  scan_step   the scan for one row per frame (serving a stream)
  join        s = x + scale silu(gate) rms(branch) post,  y = rms(s) next: from a block's result to the next block's input; `train`: also
              the gradients
x, B and C of the scan lie side by side in rows of the convolution's result, as a block hands them over, and so do their gradients.
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
        # the rows one sweep adds to a stream, between two blocks: a single short call, latency is everything
        {"name": "join_few_rows_f16", "op": "join", "rows": 37, "channels": 64, "dtype": "f16", "gate": True, "train": False},
        # all voxels of eight 64-beam frames between two blocks: serving a batch
        {"name": "join_8_frames_f16", "op": "join", "rows": 613217, "channels": 64, "dtype": "f16", "gate": True, "train": False},
        # a training batch of wide voxel rows
        {"name": "join_train_bf16", "op": "join", "rows": 240001, "channels": 128, "dtype": "bf16", "gate": True, "train": True},
        # fused LiDAR and image rows of a width that is no power of two, no gate, full precision
        {"name": "join_train_ragged_f32", "op": "join", "rows": 20011, "channels": 90, "dtype": "f32", "gate": False, "train": True},
        # one new row for each of eight streams: the serving form
        {"name": "conv_step_8_streams_f16", "op": "conv_step", "frames": 8, "channels": 160, "taps": 4, "dtype": "f16"},
        # eight whole frames: long sequences, few of them
        {"name": "conv_8_frames_f16", "op": "conv", "rows": 613217, "frames": 8, "channels": 96, "taps": 4, "dtype": "f16", "backwards": False,
         "train": False},
        # a training batch of three ragged frames, walked from their ends
        {"name": "conv_train_bf16", "op": "conv", "rows": 200003, "frames": 3, "channels": 160, "taps": 4, "dtype": "bf16", "backwards": True,
         "train": True},
        # one new row for each of eight streams: the serving form
        {"name": "scan_step_8_streams_f16", "op": "scan_step", "frames": 8, "channels": 128, "states": 16, "dtype": "f16"},
        # the rows one sweep adds to a stream: one short sequence
        {"name": "scan_short_f16", "op": "scan", "rows": 300, "frames": 1, "channels": 128, "states": 16, "dtype": "f16", "backwards": False,
         "train": False},
        # eight whole frames: long sequences, few of them
        {"name": "scan_8_frames_f16", "op": "scan", "rows": 613217, "frames": 8, "channels": 64, "states": 16, "dtype": "f16",
         "backwards": False, "train": False},
        # a training batch of three ragged frames, scanned from their ends
        {"name": "scan_train_bf16", "op": "scan", "rows": 200003, "frames": 3, "channels": 128, "states": 16, "dtype": "bf16",
         "backwards": True, "train": True},
        # a training batch of many short sequences of very different lengths (the voxels of single objects), some empty, odd widths, full precision
        {"name": "scan_train_many_short_f32", "op": "scan", "rows": 30011, "frames": 1501, "channels": 90, "states": 12, "dtype": "f32",
         "backwards": False, "train": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Channels: half the time a multiple of 16, else anything."""
    c = _log_int(rng, lo, hi)
    return max(16, c // 16 * 16) if rng.random() < 0.5 else c


def draw(rng):
    op = rng.choice(["join", "join", "conv", "conv", "conv_step", "scan", "scan", "scan", "scan_step"])
    dtype = rng.choice(["f16", "bf16", "f32"])
    train = rng.random() < 0.5
    if op == "join":
        channels = _width(rng, 8, 1024)
        return {"op": op, "rows": min(_log_int(rng, 1, 600000), 16000000 // channels), "channels": channels, "dtype": dtype,
                "gate": rng.random() < 0.7, "train": train}
    taps = rng.choice([2, 3, 4, 4, 5, 8])
    states = rng.choice([4, 8, 16, 16, 32, 64, rng.randint(1, 64)])
    if op == "conv_step":
        return {"op": op, "frames": _log_int(rng, 1, 4096), "channels": _width(rng, 8, 1024), "taps": taps, "dtype": dtype}
    if op == "scan_step":
        return {"op": op, "frames": _log_int(rng, 1, 2048), "channels": _width(rng, 8, 512), "states": states, "dtype": dtype}
    channels = _width(rng, 8, 1024 if op == "conv" else 512)
    room = 16000000 // channels if op == "conv" else (200000000 if train else 400000000) // (channels * states)
    rows = min(_log_int(rng, 1, 600000), room)
    case = {"op": op, "rows": rows, "frames": _log_int(rng, 1, max(1, rows // 8)), "channels": channels, "dtype": dtype,
            "backwards": rng.random() < 0.5, "train": train}
    return {**case, "taps": taps} if op == "conv" else {**case, "states": states}


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
    td, c, op, f32 = _TD[case["dtype"]], case["channels"], case["op"], torch.float32

    def randn(*shape, scale=1.0, shift=0.0, to=td):
        return (torch.randn(shape, generator=g, device="cuda") * scale + shift).to(to)

    n = case["frames"] if op.endswith("step") else case["rows"]
    s = {}
    if op == "join":
        s["x"] = randn(n, c)
        # a block's rows, of different magnitude; every 64th a row of zeros (a voxel that nothing reached)
        s["branch"] = (randn(n, c, to=f32) * torch.exp(torch.randn((n, 1), generator=g, device="cuda"))).to(td)
        s["branch"][5::64] = 0
        if case["gate"]:
            s["gate"] = randn(n, c)
        s["post"], s["next"] = randn(c, scale=0.2, shift=1.0, to=f32), randn(c, scale=0.2, shift=1.0, to=f32)
        s["scale"] = randn(1, scale=0.05, shift=0.5, to=f32)
        if case["train"]:
            s["dsum"], s["dy"] = randn(n, c), randn(n, c)
        return s
    if not op.endswith("step"):
        off = _offsets(n, case["frames"], seed)
        s["longest"] = int(np.max(np.diff(off)))
        s["offsets"] = torch.from_numpy(off.astype(np.int32)).cuda()
    if op.startswith("conv"):
        k = case["taps"]
        s["x"] = randn(n, c)
        s["w"], s["bias"] = randn(k, c, scale=k ** -0.5, to=f32), randn(c, scale=0.1, to=f32)
        s["before"] = randn(case["frames"], k - 1, c).float()               # rows of the stream so far
        if case.get("train"):
            s["dy"], s["dlast"] = randn(n, c), randn(case["frames"], k - 1, c, to=f32)
        return s
    m = case["states"]
    wide = randn(n, c + 2 * m)
    s["x"], s["b"], s["c"] = wide[:, :c], wide[:, c:c + m], wide[:, c + m:]
    # steps of 0.001 to 0.1, a few that forget everything; decays of 1 to `states` a unit of step; states of a sequence under way
    step = torch.exp(torch.rand(c, generator=g, device="cuda") * math.log(100) + math.log(0.001))
    s["dt"], s["dt_bias"] = randn(n, c, scale=0.5), torch.log(torch.expm1(step))
    s["dt"][::37] = randn(*s["dt"][::37].shape, scale=8.0)
    s["a"] = -torch.arange(1, m + 1, device="cuda") * torch.exp(randn(c, m, scale=0.1, to=f32))
    s["skip"] = randn(c, scale=0.2, shift=1.0, to=f32)
    s["h0"] = randn(case["frames"], c, m, to=f32)
    if case.get("train"):
        s["dy"], s["dlast"] = randn(n, c), randn(case["frames"], c, m, to=f32)
    return s


@functools.lru_cache(maxsize=None)
def _context():
    from paper_2507_04123_amd import binding as B
    return B.Context(1, 1, 1)


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    return {**s, **_held(case, s)} if own else s


def _held(case, s):
    """What a program that calls the library keeps beside its inputs: the context and its buffers."""
    from paper_2507_04123_amd import binding as B
    ctx, c, op, train = _context(), case["channels"], case["op"], case.get("train", False)
    dt = {"f32": B.F32, "f16": B.F16, "bf16": B.BF16}[case["dtype"]]
    n = s["x"].shape[0]

    def rows(width=c):
        return torch.empty((n, width), dtype=s["x"].dtype, device="cuda")

    def work(size):
        return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")

    new = {"ctx": ctx, "type": dt, "y": rows()}
    if op == "join":
        new["sum"] = rows()
        if train:
            new.update(dx=rows(), dbranch=rows(), dpost=torch.empty_like(s["post"]), dscale=torch.empty_like(s["scale"]),
                       dnext=torch.empty_like(s["next"]), work=work(ctx.gated_residual_work(dt, n, c)))
            if case["gate"]:
                new["dgate"] = rows()
    elif op == "conv_step":
        new["kept"] = torch.empty_like(s["before"])
    elif op == "conv":
        new["last"] = torch.empty_like(s["before"])
        if train:
            new.update(dx=rows(), dw=torch.empty_like(s["w"]), dbias=torch.empty_like(s["bias"]), dbefore=torch.empty_like(s["before"]),
                       work=work(ctx.causal_conv_work(dt, n, c, case["taps"])))
    elif op == "scan_step":
        new["h"] = torch.empty_like(s["h0"])
    else:
        m = case["states"]
        new.update(last=torch.empty_like(s["h0"]), work=work(ctx.selective_scan_work(dt, n, c, m)))
        if train:
            wide = rows(c + 2 * m)
            new.update(dx=wide[:, :c], db=wide[:, c:c + m], dc=wide[:, c + m:], ddt=rows(), da=torch.empty_like(s["a"]),
                       dskip=torch.empty_like(s["skip"]), ddt_bias=torch.empty_like(s["dt_bias"]), dh0=torch.empty_like(s["h0"]))
    return new


# --------------------------------------------------------------------------------------------------------------
# run
# --------------------------------------------------------------------------------------------------------------

def run(state):
    return _RUN[state["case"]["op"], own](state)


def _pick(s, *names):
    return {k: s[k] for k in names if k in s}


def _join_own(s):
    s["ctx"].gated_residual(s["type"], s["x"], s["branch"], s["post"], s["scale"], s["sum"], _EPS, gate=s.get("gate"), next_gain=s["next"],
                            y=s["y"])
    if s["case"]["train"]:
        s["ctx"].gated_residual_backward(s["type"], s["x"], s["branch"], s["post"], s["scale"], _EPS, s["dsum"], s["dx"], s["dbranch"],
                                         s["dpost"], s["dscale"], s["work"], gate=s.get("gate"), dgate=s.get("dgate"), next_gain=s["next"],
                                         dy=s["dy"], dnext=s["dnext"])
    return _pick(s, "sum", "y", "dx", "dbranch", "dgate", "dpost", "dscale", "dnext")


def _join_plain(s):
    td, x, v = s["x"].dtype, s["x"].float(), s["branch"].float()
    rv = torch.rsqrt((v * v).mean(1, keepdim=True) + _EPS)
    vh = v * rv
    if "gate" in s:
        z = s["gate"].float()
        on = 1 / (1 + torch.exp(-z))
        act, slope = z * on, on * (1 + z * (1 - on))
    else:
        act = torch.ones_like(v)
    total = x + s["scale"] * (act * vh * s["post"])
    rs = torch.rsqrt((total * total).mean(1, keepdim=True) + _EPS)
    th = total * rs
    out = {"sum": total.to(td), "y": (th * s["next"]).to(td)}
    if "dy" in s:
        dy = s["dy"].float()
        q = dy * s["next"]
        ds = s["dsum"].float() + rs * (q - th * (q * th).mean(1, keepdim=True))
        d = ds * act * s["scale"] * s["post"]
        out.update(dx=ds.to(td), dbranch=(rv * (d - vh * (d * vh).mean(1, keepdim=True))).to(td))
        if "gate" in s:
            out["dgate"] = (ds * s["scale"] * vh * s["post"] * slope).to(td)
        col = (ds * act * vh).sum(0)
        out.update(dpost=s["scale"] * col, dscale=(col * s["post"]).sum(0, keepdim=True), dnext=(dy * th).sum(0))
    return out


def _conv_own(s):
    back = s["case"]["backwards"]
    s["ctx"].causal_conv(s["type"], s["x"], s["w"], s["offsets"], s["y"], bias=s["bias"], silu=True, backwards=back, before=s["before"],
                         last=s["last"])
    if s["case"]["train"]:
        s["ctx"].causal_conv_backward(s["type"], s["x"], s["w"], s["offsets"], s["dy"], s["dx"], s["dw"], s["work"], bias=s["bias"],
                                      dbias=s["dbias"], silu=True, backwards=back, before=s["before"], dlast=s["dlast"], dbefore=s["dbefore"])
    return _pick(s, "y", "last", "dx", "dw", "dbias", "dbefore")


def _ends(off, n, back):
    """First and last row of every sequence and whether it has any, counted in the direction of the walk."""
    first, last = off[:-1], off[1:] - 1
    some = last >= first
    return (n - 1 - last, n - 1 - first, some) if back else (first, last, some)


def _conv_plain(s):
    td, w, k, n = s["x"].dtype, s["w"], s["case"]["taps"], s["x"].shape[0]
    turn = (lambda t: t.flip(0)) if s["case"]["backwards"] else (lambda t: t)
    x = turn(s["x"].float())
    off = s["offsets"].long()
    first, end, some = _ends(off, n, s["case"]["backwards"])
    length = off[1:] - off[:-1]
    seq = turn(torch.repeat_interleave(torch.arange(len(length), device="cuda"), length))
    row = torch.arange(n, device="cuda")
    place = row - first[seq]                                  # of a row in its sequence
    z = s["bias"] + w[0] * x
    taps = [x]
    for j in range(1, k):
        at = (place - j + k - 1).clamp(0, k - 2)
        taps.append(torch.where((place >= j)[:, None], x[(row - j).clamp(min=0)], s["before"][seq, at]))
        z = z + w[j] * taps[j]
    on = 1 / (1 + torch.exp(-z))
    out = {"y": turn(z * on).to(td), "last": torch.empty_like(s["before"])}
    for j in range(k - 1):                                    # the rows kept, oldest first
        at = length - (k - 1) + j
        out["last"][:, j] = torch.where((at >= 0)[:, None], x[(first + at).clamp(0, n - 1)], s["before"][torch.arange(len(length), device="cuda"),
                                                                                                         (at + k - 1).clamp(0, k - 2)])
    if "dy" not in s:
        return out
    dz = turn(s["dy"].float()) * on * (1 + z * (1 - on))
    dx, left = w[0] * dz, end[seq] - row                      # rows behind a row in its sequence
    for j in range(1, k):
        dx = dx + torch.where((left >= j)[:, None], w[j] * dz[(row + j).clamp(max=n - 1)], 0)
    dbefore = torch.zeros_like(s["before"])
    for i in range(k - 1):                                    # row i - (k - 1) of a sequence
        for j in range(k - 1 - i, k):
            at = i - (k - 1) + j
            dbefore[:, i] += torch.where((at < length)[:, None], w[j] * dz[(first + at).clamp(0, n - 1)], 0)
    for j in range(k - 1):
        at = length - (k - 1) + j
        inside = at >= 0
        dx[(first + at)[inside]] += s["dlast"][inside, j]
        dbefore[torch.nonzero(~inside)[:, 0], (at + k - 1)[~inside]] += s["dlast"][~inside, j]
    out.update(dx=turn(dx).to(td), dw=torch.stack([(dz * t).sum(0) for t in taps]), dbias=dz.sum(0), dbefore=dbefore)
    return out


def _conv_step_own(s):
    s["ctx"].causal_conv_step(s["type"], s["x"], s["w"], s["before"], s["kept"], s["y"], bias=s["bias"], silu=True)
    return _pick(s, "y", "kept")


def _conv_step_plain(s):
    rows = torch.cat([s["before"], s["x"].float()[:, None]], 1)
    z = (rows * s["w"].flip(0)).sum(1) + s["bias"]
    return {"y": (z / (1 + torch.exp(-z))).to(s["x"].dtype), "kept": rows[:, 1:].contiguous()}


def _scan_own(s):
    back = s["case"]["backwards"]
    s["ctx"].selective_scan(s["type"], s["x"], s["dt"], s["a"], s["b"], s["c"], s["offsets"], s["y"], s["work"], skip=s["skip"],
                            dt_bias=s["dt_bias"], backwards=back, h0=s["h0"], last=s["last"])
    if s["case"]["train"]:
        s["ctx"].selective_scan_backward(s["type"], s["x"], s["dt"], s["a"], s["b"], s["c"], s["offsets"], s["dy"], s["dx"], s["ddt"], s["da"],
                                         s["db"], s["dc"], s["work"], skip=s["skip"], dskip=s["dskip"], dt_bias=s["dt_bias"],
                                         ddt_bias=s["ddt_bias"], backwards=back, h0=s["h0"], dlast=s["dlast"], dh0=s["dh0"])
    return _pick(s, "y", "last", "dx", "ddt", "da", "db", "dc", "dskip", "ddt_bias", "dh0")


def _softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))


def _doubling(a, b, longest):
    """u_t = a_t u_{t-1} + b_t by doubling; a_t = 0 where a sequence of at most `longest` rows begins."""
    step = 1
    while step < longest:
        b = torch.cat([b[:step], b[step:] + a[step:] * b[:-step]])
        a = torch.cat([a[:step], a[step:] * a[:-step]])
        step *= 2
    return b


def _scan_plain(s):
    td, n, back = s["x"].dtype, s["x"].shape[0], s["case"]["backwards"]
    turn = (lambda t: t.flip(0)) if back else (lambda t: t)
    x, v, b, c = (turn(s[k].float()) for k in ("x", "dt", "b", "c"))
    v = v + s["dt_bias"]
    first, end, some = _ends(s["offsets"].long(), n, back)
    first, end = first[some], end[some]
    d = _softplus(v)
    dx_ = d * x
    keep = torch.exp(d[:, :, None] * s["a"])
    add = dx_[:, :, None] * b[:, None]
    add[first] += keep[first] * s["h0"][some]
    factor = keep.clone()
    factor[first] = 0
    h = _doubling(factor, add, s["longest"])
    last = s["h0"].clone()
    last[some] = h[end]
    out = {"y": turn((h * c[:, None]).sum(2) + s["skip"] * x).to(td), "last": last}
    if "dy" not in s:
        return out
    del add
    dy = turn(s["dy"].float())
    flow = dy[:, :, None] * c[:, None]
    flow[end] += s["dlast"][some]
    factor = torch.cat([factor[1:], torch.zeros_like(factor[:1])])           # the factor of the row behind, none behind a sequence's last
    g = _doubling(factor.flip(0), flow.flip(0), s["longest"]).flip(0)
    del factor, flow
    out["dc"] = turn((dy[:, :, None] * h).sum(1)).to(td)
    out["db"] = turn((g * dx_[:, :, None]).sum(1)).to(td)
    prev = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    prev[first] = s["h0"][some]
    out["dh0"] = s["dlast"].clone()
    out["dh0"][some] = (keep * g)[first]
    gb = (g * b[:, None]).sum(2)
    through = g * keep * prev                                                # what reaches the exponent
    dd = (through * s["a"]).sum(2) + gb * x
    dv = dd / (1 + torch.exp(-v))
    out.update(dx=turn(s["skip"] * dy + d * gb).to(td), ddt=turn(dv).to(td), da=(through * d[:, :, None]).sum(0), dskip=(dy * x).sum(0),
               ddt_bias=dv.sum(0))
    return out


def _scan_step_own(s):
    s["ctx"].selective_scan_step(s["type"], s["x"], s["dt"], s["a"], s["b"], s["c"], s["h0"], s["h"], s["y"], skip=s["skip"],
                                 dt_bias=s["dt_bias"])
    return _pick(s, "y", "h")


def _scan_step_plain(s):
    x, b, c = (s[k].float() for k in ("x", "b", "c"))
    d = _softplus(s["dt"].float() + s["dt_bias"])
    h = torch.exp(d[:, :, None] * s["a"]) * s["h0"] + (d * x)[:, :, None] * b[:, None]
    return {"y": ((h * c[:, None]).sum(2) + s["skip"] * x).to(s["x"].dtype), "h": h}


_RUN = {("join", True): _join_own, ("join", False): _join_plain, ("conv", True): _conv_own, ("conv", False): _conv_plain,
        ("conv_step", True): _conv_step_own, ("conv_step", False): _conv_step_plain, ("scan", True): _scan_own, ("scan", False): _scan_plain,
        ("scan_step", True): _scan_step_own, ("scan_step", False): _scan_step_plain}


# --------------------------------------------------------------------------------------------------------------
# work, exact
# --------------------------------------------------------------------------------------------------------------

def work(case):
    size, c, train, op = _BYTES[case["dtype"]], case["channels"], case.get("train", False), case["op"]
    n, frames = case.get("rows", 0), case.get("frames", 0)
    if op == "join":
        gate = bool(case["gate"])
        rows = 4 + gate + (4 + gate if train else 0)          # x, branch, gate; sum, y; dsum, dy, dx, dbranch, dgate
        return {"bytes": rows * n * c * size + (20 if train else 8) * c, "flops": (60 if train else 20) * n * c}
    if op == "conv_step":
        k = case["taps"]
        return {"bytes": frames * c * (2 * size + 8 * (k - 1)) + 4 * (k + 1) * c, "flops": (2 * k + 5) * frames * c}
    if op == "conv":
        k = case["taps"]
        states = (4 if train else 2) * frames * (k - 1) * c * 4              # before, last, dlast, dbefore
        return {"bytes": (4 if train else 2) * n * c * size + states + (8 if train else 4) * (k + 1) * c,
                "flops": ((6 * k + 16) if train else (2 * k + 5)) * n * c}
    m = case["states"]
    if op == "scan_step":
        return {"bytes": frames * (3 * c + 2 * m) * size + frames * c * m * 8 + 4 * c * (m + 2), "flops": 7 * frames * c * m}
    rows = (6 * c + 4 * m if train else 3 * c + 2 * m) * n * size            # x, dt, y, B, C; dy, dx, ddt, dB, dC
    return {"bytes": rows + (4 if train else 2) * frames * c * m * 4 + (8 if train else 4) * c * (m + 2), "flops": (24 if train else 7) * n * c * m}


def exact(case, seed):
    s = _inputs(case, seed)
    v = {k: t.double() if torch.is_tensor(t) and t.is_floating_point() else t for k, t in s.items()}
    if case["op"] == "join":
        return _join_exact(case, v)
    if case["op"].startswith("conv"):
        return _conv_exact(case, v)
    return _scan_exact(case, v)


def _grads(out, wanted, v, losses):
    """Adds the gradients d<name> of the sum of <output, its given gradient>."""
    sum((y * dy).sum() for y, dy in losses).backward()
    out.update({"d" + k: v[k].grad for k in wanted})
    return {k: t.detach() for k, t in out.items()}


def _join_exact(case, v):
    wanted = [k for k in ("x", "branch", "gate", "post", "scale", "next") if k in v]
    for k in wanted:
        v[k].requires_grad_(case["train"])
    t = v["branch"] / torch.sqrt(torch.mean(v["branch"] ** 2, 1, keepdim=True) + _EPS) * v["post"]
    if case["gate"]:
        t = t * (v["gate"] * torch.sigmoid(v["gate"]))
    total = v["x"] + v["scale"] * t
    y = total / torch.sqrt(torch.mean(total ** 2, 1, keepdim=True) + _EPS) * v["next"]
    out = {"sum": total, "y": y}
    return _grads(out, wanted, v, [(total, v["dsum"]), (y, v["dy"])]) if case["train"] else out


def _conv_exact(case, v):
    """Every sequence with its rows before written in front of it: a convolution of that list."""
    k, c, frames = case["taps"], case["channels"], case["frames"]
    train = case.get("train", False)
    if case["op"] == "conv_step":
        off, back = np.arange(frames + 1), False
    else:
        off, back = v["offsets"].cpu().numpy().astype(np.int64), case["backwards"]
    wanted = ("x", "w", "bias", "before")
    for name in wanted:
        v[name].requires_grad_(train)
    source, place, kept = [], np.empty(off[-1], np.int64), []                # rows of [before; x] in list order; where a row's result lies
    at = 0
    for i in range(frames):
        rows = np.arange(off[i], off[i + 1])
        rows = rows[::-1] if back else rows
        source.append(np.concatenate([np.arange(i * (k - 1), (i + 1) * (k - 1)), frames * (k - 1) + rows]))
        place[rows] = at + k - 1 + np.arange(len(rows))
        at += k - 1 + len(rows)
        kept.append(np.arange(at - (k - 1), at))
    everything = torch.cat([v["before"].reshape(-1, c), v["x"]])[torch.from_numpy(np.concatenate(source)).cuda()]
    place = torch.from_numpy(place).cuda()
    z = v["bias"] + sum(v["w"][j] * everything[place - j] for j in range(k))
    y, last = z * torch.sigmoid(z), everything[torch.from_numpy(np.concatenate(kept)).cuda()].reshape(frames, k - 1, c)
    if case["op"] == "conv_step":
        return {"y": y, "kept": last}
    out = {"y": y, "last": last}
    return _grads(out, wanted, v, [(y, v["dy"]), (last, v["dlast"])]) if train else out


def _scan_exact(case, v):
    """Row after row, as the definition says, side by side in pieces of as many rows: once from zero, for what each piece makes of a state, and once
    from the state that reaches it."""
    c, m, frames, train = case["channels"], case["states"], case["frames"], case.get("train", False)
    back = case.get("backwards", False)
    off = np.arange(frames + 1) if case["op"] == "scan_step" else v["offsets"].cpu().numpy().astype(np.int64)
    n, length = int(off[-1]), np.diff(off)
    size = 1
    while size * size * 4 < max(1, length.max()) and size < 256:
        size *= 2
    pieces, start, count = [], [], -(-length // size)                        # rows of every piece in the order of the walk, -1 behind the last
    for i in range(frames):
        rows = np.arange(off[i], off[i + 1])
        rows = rows[::-1] if back else rows
        padded = np.full(count[i] * size, -1, np.int64)
        padded[:len(rows)] = rows
        pieces.append(padded.reshape(-1, size))
        start.append(sum(count[:i]) if i < 2 else start[-1] + count[i - 1])
    pieces = torch.from_numpy(np.concatenate(pieces)).cuda()
    there = (pieces >= 0).double()[:, :, None]
    place = pieces.clamp(min=0)
    d = torch.nn.functional.softplus(v["dt"] + v["dt_bias"], beta=1, threshold=100)
    a, gain = v["a"], d * v["x"]

    def chained(begin, decay, made, backwards):
        """The state that reaches every piece, and the one behind each sequence."""
        reach, behind = torch.zeros_like(made), begin.clone()
        most = int(count.max()) if len(count) else 0
        starts, counts = torch.tensor(start).cuda(), torch.from_numpy(count).cuda()
        for j in range(most):
            live = counts > j
            at = starts[live] + (counts[live] - 1 - j if backwards else j)
            reach[at] = behind[live]
            behind[live] = decay[at] * behind[live] + made[at]
        return reach, behind

    def keep(j):
        return torch.exp((d[place[:, j]] * there[:, j])[:, :, None] * a)

    def add(j):
        return (gain[place[:, j]] * there[:, j])[:, :, None] * v["b"][place[:, j]][:, None]

    def walked(h, visit=None):
        for j in range(size):
            before, h = h, keep(j) * h + add(j)
            if visit:
                visit(j, before, h)
        return h

    zero = torch.zeros((len(pieces), c, m), dtype=torch.float64, device="cuda")
    total = (d[place] * there).sum(1)
    decay = torch.exp(total[:, :, None] * a)
    h_in, last = chained(v["h0"], decay, walked(zero), False)
    y = torch.zeros((n, c), dtype=torch.float64, device="cuda")
    befores, afters = [], []

    def put(to, j, value):
        live = pieces[:, j] >= 0
        to[pieces[live, j]] = value[live]

    def seen(j, before, h):
        put(y, j, (h * v["c"][place[:, j]][:, None]).sum(2))
        if train:
            befores.append(before)
            afters.append(h)

    walked(h_in, seen)
    out = {"y": y + v["skip"] * v["x"], "h" if case["op"] == "scan_step" else "last": last}
    if not train:
        return out

    def back_walked(g, visit=None):
        """g: what flows from behind into the state after the row (the row's own share not in it)."""
        for j in reversed(range(size)):
            own_g = g + (v["dy"][place[:, j]] * there[:, j])[:, :, None] * v["c"][place[:, j]][:, None]
            if visit:
                visit(j, own_g)
            g = keep(j) * own_g
        return g

    g_in, dh0 = chained(v["dlast"], decay, back_walked(zero), True)
    out.update(dx=v["skip"] * v["dy"], ddt=torch.zeros_like(y), da=torch.zeros_like(a), db=torch.zeros_like(v["b"]), dc=torch.zeros_like(v["c"]),
               dskip=(v["dy"] * v["x"]).sum(0), dh0=dh0)

    def back_seen(j, g):
        rows, live = place[:, j], there[:, j]
        put(out["dc"], j, (v["dy"][rows][:, :, None] * afters[j]).sum(1))
        put(out["db"], j, (g * gain[rows][:, :, None]).sum(1))
        gb, through = (g * v["b"][rows][:, None]).sum(2), g * keep(j) * befores[j]
        put(out["dx"], j, out["dx"][rows] + d[rows] * gb)
        put(out["ddt"], j, ((through * a).sum(2) + gb * v["x"][rows]) * torch.sigmoid((v["dt"] + v["dt_bias"])[rows]))
        out["da"] += (through * (d[rows] * live)[:, :, None]).sum(0)

    back_walked(g_in, back_seen)
    out["ddt_bias"] = out["ddt"].sum(0)
    return out
