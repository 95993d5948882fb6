"""Thousands of sequences, some without rows: the search for a row's sequence narrows more than once, and the kept rows and states of more sequences than the launch has
threads for are written in turns."""
import numpy as np
import pytest

from paper_2507_04123_amd import binding as B

import test_gpu_causal_conv as conv
import test_gpu_selective_scan as scan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(1, 1, 1)
    yield c
    c.status_sync()
    c.close()


def _lens(count):
    lens = np.random.RandomState(3).choice([0, 0, 1, 1, 2, 3, 4, 9], count)
    lens[100:400] = 0
    return [int(v) for v in lens]


# 6000 sequences of 96 channels: 576 000 kept columns for the 524 288 threads that write them
@pytest.mark.parametrize("dtype,taps,backwards", [("f32", 3, False), ("f16", 4, True), ("bf16", 2, False)])
def test_conv(ctx, dtype, taps, backwards):
    lens = _lens(6000)
    assert len(lens) * 96 > 2048 * 256 and len(lens) > 4096
    conv._check(ctx, dtype, lens, 96, taps, "packed", True, backwards)


@pytest.mark.parametrize("dtype,m,backwards", [("f32", 5, True), ("f16", 16, False), ("bf16", 4, True)])
def test_scan(ctx, dtype, m, backwards):
    scan._check(ctx, dtype, _lens(20000 if m == 4 else 6000), 6, m, "packed", backwards)
