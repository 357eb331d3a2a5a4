"""Pins of the oracle's norms of queries and keys with their rotation: what a rotation keeps, relative positions, complex
numbers, finite differences."""
import numpy as np
import pytest

from oracle import ops as O

RNG = np.random.default_rng(3)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("width,rotated", [(8, 8), (10, 6), (7, 4), (16, 0)])
def test_rotation(width, rotated, neighbours):
    table = O.rotary_table(50, rotated, base=100.0)
    v, at = RNG.standard_normal((5, 3, width)), np.array([0, 1, 7, 30, 49])
    y = O.rotate(v, table, at, neighbours)
    assert np.allclose((y ** 2).sum(-1), (v ** 2).sum(-1), rtol=1e-13)
    assert np.array_equal(y[0], v[0]) and np.array_equal(y[..., rotated:], v[..., rotated:])     # position 0 turns nothing
    assert np.allclose(O.rotate(y, table, at, neighbours, back=True), v, atol=1e-14)
    p = rotated // 2
    a, b = (v[..., :rotated:2], v[..., 1:rotated:2]) if neighbours else (v[..., :p], v[..., p:rotated])
    z = (a + 1j * b) * np.exp(1j * at[:, None] * 100.0 ** (-np.arange(p) / max(1, p)))[:, None]
    got = (y[..., :rotated:2], y[..., 1:rotated:2]) if neighbours else (y[..., :p], y[..., p:rotated])
    assert np.allclose(got[0], z.real, atol=1e-13) and np.allclose(got[1], z.imag, atol=1e-13)


def test_scores_depend_on_relative_positions_only():
    table = O.rotary_table(100, 12)
    q, k = RNG.standard_normal((1, 1, 12)), RNG.standard_normal((1, 1, 12))
    score = lambda i, j: (O.rotate(q, table, [i]) * O.rotate(k, table, [j])).sum()
    assert np.isclose(score(40, 33), score(97, 90), rtol=1e-12) and not np.isclose(score(40, 33), score(40, 34), rtol=1e-3)


def test_norm_gives_unit_scale_and_positions_outside_the_table_nan():
    X = RNG.standard_normal((64, 6 * 16)) * 7
    y = O.qk_norm_fwd(X, None, 16, 0.0).reshape(64, 6, 16)
    assert np.allclose((y ** 2).mean(-1), 1, rtol=1e-12)
    y = O.qk_norm_fwd(X[:3], None, 16, 0.0, O.rotary_table(10, 8), np.array([-1, 9, 10])).reshape(3, 6, 16)
    assert np.isnan(y[[0, 2], :, :8]).all() and np.isfinite(y[1]).all() and np.isfinite(y[:, :, 8:]).all()


@pytest.mark.parametrize("neighbours", [False, True])
def test_gradients_are_finite_differences(neighbours):
    width, rows, heads = 10, 4, 3
    X, w, G = RNG.standard_normal((rows, heads * width)), RNG.standard_normal(width), RNG.standard_normal((rows, heads * width))
    table, at = O.rotary_table(20, 6, base=10.0), np.array([3, 0, 19, 7])
    f = lambda X_, w_: (G * O.qk_norm_fwd(X_, w_, width, 1e-3, table, at, neighbours)).sum()
    dX, dw = O.qk_norm_bwd(X, w, G, width, 1e-3, 1.0, 1.0, table, at, neighbours)
    h = 1e-6
    for i in range(rows):
        for j in range(heads * width):
            E = np.zeros_like(X)
            E[i, j] = h
            assert abs((f(X + E, w) - f(X - E, w)) / (2 * h) - dX[i, j]) < 1e-7
    for j in range(width):
        e = np.zeros(width)
        e[j] = h
        assert abs((f(X, w + e) - f(X, w - e)) / (2 * h) - dw[j]) < 1e-7
    assert np.allclose(O.qk_norm_bwd(X, w, G, width, 1e-3, 2.0, 0.5, table, at, neighbours)[0], 2 * dX)
