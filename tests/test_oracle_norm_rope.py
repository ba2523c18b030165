"""Pins of the oracle of the norms and rotations of Q and K: closed forms, complex numbers, differences (CPU only)."""
import numpy as np
import pytest

from oracle import paro_norm_rope as on


def _table(grid, dims, pos=None):
    pos = np.concatenate([np.arange(n) for n in grid]).astype(np.float64) if pos is None else pos
    freq = np.concatenate([100.0 ** (-np.arange(0, k, 2) / max(k, 1)) for k in dims])
    return on.rope_table(grid, dims, pos, freq), pos, freq


@pytest.mark.parametrize("halves", [0, 1])
def test_a_pair_turns_by_coordinate_times_frequency(halves):
    grid, dims, d = (2, 3, 4), (4, 2, 6), 16  # 6 pairs turn, 2 do not
    table, pos, freq = _table(grid, dims)
    cos, sin = on.token_angles(grid, 1, d, dims, table)
    x = np.random.default_rng(0).standard_normal((25, d))
    y = on.turn(x, cos, sin, halves)
    a, b = on.pair_channels(d, halves)
    axis = [0, 0, 1, 2, 2, 2]
    for n in range(24):
        coord = (n // 12, n // 4 % 3, n % 4)
        for p in range(8):
            z = complex(x[n, a[p]], x[n, b[p]])
            if p < 6:
                z *= np.exp(1j * coord[axis[p]] * freq[p])
            assert abs(complex(y[n, a[p]], y[n, b[p]]) - z) <= 2**-23 * abs(z) + 1e-15  # the table is float32
    assert np.array_equal(y[24], x[24])  # a text token
    back = on.turn(y, cos, sin, halves, inverse=True)
    assert np.allclose(back, x, rtol=0, atol=1e-6)


def test_products_depend_on_the_difference_of_positions():
    d, dims = 8, (2, 2, 4)
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, d))
    dots = []
    for start in (0.0, 17.0, -5.5):
        grid = (2, 2, 2)
        pos = np.concatenate([start + np.arange(2.0)] * 3)
        table, _, _ = _table(grid, dims, pos)
        cos, sin = on.token_angles(grid, 0, d, dims, table)
        dots.append(on.turn(q, cos[6], sin[6], 0) @ on.turn(k, cos[1], sin[1], 0))
    assert np.ptp(dots) < 1e-6 * np.abs(dots).max() + 1e-6


def test_what_does_not_turn_is_left_alone_beside_an_infinity():
    y = on.turn(np.array([[1.0, np.inf, np.nan, 2.0]]), np.ones((1, 2)), np.zeros((1, 2)), 0)
    assert y[0, 0] == 1.0 and np.isinf(y[0, 1]) and np.isnan(y[0, 2]) and y[0, 3] == 2.0


def test_norms_of_hand_worked_rows():
    h, r = on.normed(np.array([[3.0, 4.0, 0.0, 0.0]]), "rms", 0.0)
    assert np.allclose(h, [[1.2, 1.6, 0, 0]]) and np.allclose(r, 1 / 2.5)
    h, r = on.normed(np.array([[1.0, 3.0]]), "layer", 3.0)
    assert np.allclose(h, [[-0.5, 0.5]]) and np.allclose(r, 0.5)
    assert np.array_equal(on.normed(np.zeros((1, 4)), "rms", 1e-6)[0], np.zeros((1, 4)))
    w = on.per_token(np.ones(2), np.full(2, 5.0), 1, 3)
    assert np.array_equal(w, [[1, 1], [5, 5], [5, 5]])


@pytest.mark.parametrize("kind", ["none", "rms", "layer"])
@pytest.mark.parametrize("halves", [0, 1])
def test_gradients_are_the_differences(kind, halves):
    grid, dims, d, eps = (1, 2, 2), (0, 2, 4), 8, 0.1
    table, _, _ = _table(grid, dims)
    cos, sin = on.token_angles(grid, 1, d, dims, table)
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 5, d))
    w, b = 1 + 0.3 * rng.standard_normal((5, d)), rng.standard_normal((5, d))
    loss = lambda x, w, b: np.sum(on.norm_rope(x, kind, eps, w, b, cos, sin, halves) * dy)
    dx, dw, db = on.norm_rope_backward(x, dy, kind, eps, w, cos, sin, halves)
    step = 1e-6
    for grad, i in ((dx, 0), (dw, 1), (db, 2)):
        if grad is None or (i == 2 and kind != "layer"):
            continue
        for at in np.ndindex(x.shape):
            args = [x, w, b]
            hi, lo = np.array(args[i]), np.array(args[i])
            hi[at] += step
            lo[at] -= step
            diff = (loss(*args[:i], hi, *args[i + 1:]) - loss(*args[:i], lo, *args[i + 1:])) / (2 * step)
            assert abs(diff - grad[at]) < 1e-7 * (1 + abs(grad[at])), (i, at)
