"""The oracle of the sequence operators against closed forms, library routines and differences (no GPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import sequence as S


def _r(*shape, seed=0):
    return np.random.RandomState(seed).standard_normal(shape)


def _difference(f, args, k, seed, step=1e-5):
    """(directional difference of f along a random direction of args[k], that direction)"""
    d = _r(*args[k].shape, seed=seed)
    up, down = list(args), list(args)
    up[k], down[k] = args[k] + step * d, args[k] - step * d
    return (f(*up) - f(*down)) / (2 * step), d


# central differences: error step^2 of third derivatives (of order one here) plus 1e-16 / step: 1e-9 relative, 1e-6 asked
def _check(f, args, grads, which):
    for k, g in zip(which, grads):
        num, d = _difference(f, args, k, 40 + k)
        assert abs(num - (g * d).sum()) <= 1e-6 * (1 + abs(num)), k


def test_layernorm_is_the_library_routine_and_its_gradient_the_difference():
    x, gamma, beta, dy = _r(7, 12, seed=1) * 3 + 1, _r(12, seed=2), _r(12, seed=3), _r(7, 12, seed=4)
    ref = torch.nn.functional.layer_norm(torch.from_numpy(x), (12,), torch.from_numpy(gamma), torch.from_numpy(beta), 1e-5)
    assert np.allclose(S.layernorm(x, gamma, beta, 1e-5), ref.numpy(), rtol=1e-12, atol=1e-12)
    _check(lambda *a: (S.layernorm(*a, 1e-5) * dy).sum(), (x, gamma, beta), S.layernorm_backward(x, gamma, 1e-5, dy), (0, 1, 2))


@pytest.mark.parametrize("backwards", [False, True])
def test_recurrence_closed_form_and_gradients(backwards):
    off = [0, 4, 4, 5, 12]
    x, gate, h0 = _r(12, 3, seed=1), _r(12, 3, seed=2) * 2, _r(4, 3, seed=3)
    y, last = S.recurrence(x, gate, off, h0, backwards)
    a = 1 / (1 + np.exp(-gate))
    rows = list(range(5, 12))[::-1] if backwards else list(range(5, 12))
    h = h0[3] * np.prod(a[rows], axis=0)                     # the last state as a sum over its sequence's rows
    for i, t in enumerate(rows):
        h = h + (1 - a[t]) * x[t] * np.prod(a[rows[i + 1:]], axis=0)
    assert np.allclose(last[3], h, rtol=1e-12) and np.allclose(y[rows[-1]], h, rtol=1e-12)
    assert np.array_equal(last[1], h0[1])
    assert np.allclose(S.recurrence(x, np.full_like(x, 60.0), off, h0, backwards)[1], h0, atol=1e-20 + 1e-24)   # open gates keep the state
    dy, dlast = _r(12, 3, seed=5), _r(4, 3, seed=6)

    def loss(x, gate, h0):
        y, last = S.recurrence(x, gate, off, h0, backwards)
        return (y * dy).sum() + (last * dlast).sum()

    _check(loss, (x, gate, h0), S.recurrence_backward(x, gate, off, h0, dy, dlast, backwards), (0, 1, 2))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_feed_forward_activations_and_gradients(act):
    g = np.linspace(-9, 9, 101)
    lib = torch.nn.functional.silu if act == "silu" else lambda t: torch.nn.functional.gelu(t, approximate="tanh")
    assert np.allclose(S.activate(act, g)[0], lib(torch.from_numpy(g)).numpy(), rtol=1e-12, atol=1e-13)
    x, wg, wu, wd, dy = _r(5, 6, seed=1), _r(6, 9, seed=2), _r(6, 9, seed=3), _r(9, 6, seed=4), _r(5, 6, seed=5)
    _check(lambda *a: (S.ffn(act, *a) * dy).sum(), (x, wg, wu, wd), S.ffn_backward(act, x, wg, wu, wd, dy), (0, 1, 2, 3))


def test_frame_offsets_counts_rows_of_earlier_frames():
    coords = np.array([[0, 1, 1, 1], [0, 1, 1, 2], [2, 0, 0, 0], [5, 0, 0, 0]])
    assert S.frame_offsets(coords, 7).tolist() == [0, 2, 2, 3, 3, 3, 4, 4]
    assert S.frame_offsets(coords[:0], 2).tolist() == [0, 0, 0]
    assert math.isclose(S.sigmoid(np.float64(-800.0)), 0.0)
