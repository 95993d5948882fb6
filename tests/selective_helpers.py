"""What the tests of the selective state space operators share: seeded rows in several layouts, comparisons, sequences of many shapes."""
import numpy as np
import torch

from paper_2507_04123_amd import binding as B

TD = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DT = {"f32": B.F32, "f16": B.F16, "bf16": B.BF16}
TYPES = list(TD)

LENGTHS = {"one": [1], "none": [0], "empties": [0, 5, 0, 0, 7, 1, 0], "two": [2, 0, 2], "long": [2100], "around": [255, 1, 256, 257, 0, 511],
           "short": [3, 0, 1, 2, 9, 4] * 60, "ragged": [1, 700, 0, 33, 900, 2, 64, 64], "all_empty": [0] * 70, "many_empty": [0] * 70 + [9] + [0] * 200 + [40, 1]}


def draw(seed, *shape, scale=1.0, shift=0.0, dtype="f32"):
    v = torch.from_numpy(np.random.RandomState(seed).standard_normal(shape) * scale + shift)
    return v.to(TD[dtype])


def f64(t):
    return t.double().cpu().numpy()


def rows(t, how):
    """The rows `t` on the GPU: packed; a 16-byte aligned slice of wider rows; an odd slice of them."""
    t = t.cuda()
    if how == "packed":
        return t
    n, c = t.shape
    at = 16 if how == "slice" else 1
    wide = torch.full((n, (c + 2 * at + 15) // 16 * 16 + (0 if how == "slice" else 3)), 7.0, dtype=t.dtype, device="cuda")
    wide[:, at:at + c] = t
    return wide[:, at:at + c]


def like(t, how, fill=-3.0):
    return rows(torch.full(t.shape, fill, dtype=t.dtype), how)


def within(got, exp, bound, what):
    got = f64(got)
    assert got.shape == exp.shape, what
    bad = ~(np.abs(got - exp) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside, first {i}: {got[i]!r}, {exp[i]!r} +- {bound[i]:.3g}")


def work(size):
    return torch.full((max(size, 16),), 0xA5, dtype=torch.uint8, device="cuda")


def offsets(lens):
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    return off, torch.from_numpy(off.astype(np.int32)).cuda()
