"""Pins of the selective state space operators' definitions (CPU): library routines, closed forms, and differences for every gradient."""
import numpy as np
import pytest
import torch

from oracle import selective as V


def _r(seed, *shape):
    return np.random.RandomState(seed).standard_normal(shape)


OFF = np.array([0, 5, 5, 6, 17])


@pytest.mark.parametrize("taps", [2, 4, 8])
def test_conv_is_the_librarys_on_one_sequence(taps):
    x, w, bias = _r(1, 19, 6), _r(2, taps, 6), _r(3, 6)
    y, last = V.causal_conv(x, w, bias, np.array([0, 19]), np.zeros((1, taps - 1, 6)), silu=False)
    t = torch.from_numpy(x.T.copy())[None]
    e = torch.nn.functional.conv1d(torch.nn.functional.pad(t, (taps - 1, 0)), torch.from_numpy(w[::-1].T.copy())[:, None], torch.from_numpy(bias), groups=6)
    assert np.allclose(y, e[0].T.numpy(), rtol=0, atol=1e-13)
    assert np.array_equal(last[0], x[19 - (taps - 1):])


@pytest.mark.parametrize("backwards", [False, True])
def test_conv_of_a_sequence_in_two_parts_and_from_its_end(backwards):
    """A sequence cut in two goes on with the rows kept; backwards is forwards over the reversed rows."""
    x, w, bias, before = _r(1, 23, 3), _r(2, 4, 3), _r(3, 3), _r(4, 1, 3, 3)
    turn = x[::-1] if backwards else x
    whole, end = V.causal_conv(turn.copy(), w, bias, np.array([0, 23]), before)
    for cut in (1, 2, 9):
        first, mid = V.causal_conv(turn[:cut].copy(), w, bias, np.array([0, cut]), before)
        rest, last = V.causal_conv(turn[cut:].copy(), w, bias, np.array([0, 23 - cut]), mid)
        assert np.allclose(np.concatenate([first, rest]), whole, rtol=0, atol=1e-14) and np.array_equal(last, end)
    if backwards:
        y, last = V.causal_conv(x, w, bias, np.array([0, 23]), before, backwards=True)
        assert np.allclose(y[::-1], whole, rtol=0, atol=1e-14) and np.array_equal(last, end)


def test_scan_of_constant_steps_is_a_geometric_sum():
    """With the same step, B and C in every row the state after t rows is decay^t h0 + add (1 - decay^t) / (1 - decay)."""
    n, c, m = 12, 3, 4
    a, v, b = -np.abs(_r(1, c, m)) - 0.1, _r(2, c), _r(3, m)
    h0, x = _r(4, 1, c, m), np.ones((n, c))
    y, last = V.selective_scan(x, np.tile(v, (n, 1)), a, np.tile(b, (n, 1)), np.ones((n, m)), np.array([0, n]), h0, np.zeros(c), np.zeros(c))
    d = np.log(1 + np.exp(v))
    keep = np.exp(d[:, None] * a)
    for t in range(1, n + 1):
        h = keep ** t * h0[0] + d[:, None] * b * (1 - keep ** t) / (1 - keep)
        assert np.allclose(y[t - 1], h.sum(1), rtol=1e-12)
    assert np.allclose(last[0], h, rtol=1e-12)


def test_scan_hands_on_the_states_of_empty_sequences_and_resets_between_them():
    x, dt, b, c = _r(1, 17, 3), _r(2, 17, 3), _r(3, 17, 2), _r(4, 17, 2)
    a, h0, skip, bias = -np.abs(_r(5, 3, 2)), _r(6, 4, 3, 2), _r(7, 3), _r(8, 3)
    y, last = V.selective_scan(x, dt, a, b, c, OFF, h0, skip, bias)
    assert np.array_equal(last[1], h0[1])
    for s in range(4):
        lo, hi = OFF[s], OFF[s + 1]
        one, end = V.selective_scan(x[lo:hi], dt[lo:hi], a, b[lo:hi], c[lo:hi], np.array([0, hi - lo]), h0[s:s + 1], skip, bias)
        assert np.array_equal(one, y[lo:hi]) and np.array_equal(end[0], last[s])


@pytest.mark.parametrize("gate", [False, True])
def test_gated_residual_is_the_librarys_norms(gate):
    x, b, z, post, nxt = _r(1, 7, 9), _r(2, 7, 9), _r(3, 7, 9) if gate else None, _r(4, 9), _r(5, 9)
    total, y = V.gated_residual(x, b, z, post, 0.3, nxt, 1e-5)
    t = lambda v: torch.from_numpy(v)  # noqa: E731
    e = torch.nn.functional.rms_norm(t(b), (9,), t(post), 1e-5) * (torch.nn.functional.silu(t(z)) if gate else 1.0) * 0.3 + t(x)
    assert np.allclose(total, e.numpy(), rtol=0, atol=1e-13)
    assert np.allclose(y, torch.nn.functional.rms_norm(e, (9,), t(nxt), 1e-5).numpy(), rtol=0, atol=1e-13)


def _differences(loss, at, grads):
    """Every gradient along a random direction against central differences."""
    for i, k in enumerate(grads):
        d = _r(100 + i, *np.shape(at[k]))
        num = (loss({**at, k: at[k] + 1e-5 * d}) - loss({**at, k: at[k] - 1e-5 * d})) / 2e-5
        assert abs(num - (grads[k] * d).sum()) <= 1e-8 * (1 + np.abs(grads[k] * d).sum()), k


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("backwards", [False, True])
def test_conv_gradients_are_differences(silu, backwards):
    at = {"x": _r(1, 17, 4), "w": _r(2, 4, 4), "bias": _r(3, 4), "before": _r(4, 4, 3, 4)}
    dy, dlast = _r(5, 17, 4), _r(6, 4, 3, 4)

    def loss(p):
        y, last = V.causal_conv(p["x"], p["w"], p["bias"], OFF, p["before"], silu, backwards)
        return (y * dy).sum() + (last * dlast).sum()

    got = V.causal_conv_backward(at["x"], at["w"], at["bias"], OFF, at["before"], dy, dlast, silu, backwards)
    _differences(loss, at, dict(zip(at, got)))


@pytest.mark.parametrize("backwards", [False, True])
def test_scan_gradients_are_differences(backwards):
    at = {"x": _r(1, 17, 3), "dt": _r(2, 17, 3), "a": -np.abs(_r(3, 3, 5)), "b": _r(4, 17, 5), "c": _r(5, 17, 5), "h0": _r(6, 4, 3, 5), "skip": _r(7, 3),
          "dt_bias": _r(8, 3)}
    dy, dlast = _r(9, 17, 3), _r(10, 4, 3, 5)

    def loss(p):
        y, last = V.selective_scan(p["x"], p["dt"], p["a"], p["b"], p["c"], OFF, p["h0"], p["skip"], p["dt_bias"], backwards)
        return (y * dy).sum() + (last * dlast).sum()

    got = V.selective_scan_backward(*(at[k] for k in ("x", "dt", "a", "b", "c")), OFF, at["h0"], at["skip"], at["dt_bias"], dy, dlast, backwards)
    _differences(loss, at, {k: got["d" + k] for k in at})


@pytest.mark.parametrize("gate", [False, True])
def test_gated_residual_gradients_are_differences(gate):
    at = {"x": _r(1, 6, 5), "branch": _r(2, 6, 5), "gate": _r(3, 6, 5), "post": _r(4, 5), "scale": np.array([0.7]), "next": _r(5, 5)}
    dsum, dy = _r(6, 6, 5), _r(7, 6, 5)

    def args(p):
        return p["x"], p["branch"], p["gate"] if gate else None, p["post"], p["scale"], p["next"], 1e-3

    def loss(p):
        total, y = V.gated_residual(*args(p))
        return (total * dsum).sum() + (y * dy).sum()

    got = V.gated_residual_backward(*args(at), dsum, dy)
    _differences(loss, at, {k: got["d" + k] for k in at if gate or k != "gate"})
