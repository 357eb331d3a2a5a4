"""Pins of the oracle's gated hidden layer, and of the library's host helpers for it: finite differences, library silu, unit scale."""
import numpy as np
import pytest
import torch

from oracle import ops as O
from oracle import scales as S

RNG = np.random.default_rng(5)
FNS = {"gelu": (S.gelu, S.gelu_grad), "relu": (lambda z: np.maximum(z, 0.0), lambda z: (z > 0) * 1.0), "tanh": (np.tanh, lambda z: 1 - np.tanh(z) ** 2),
       "sigmoid": (lambda z: 1 / (1 + np.exp(-z)), lambda z: np.exp(-z) / (1 + np.exp(-z)) ** 2), "silu": (S.silu, S.silu_grad)}


def test_silu_is_the_library_function():
    z = np.linspace(-30, 30, 601)
    t = torch.from_numpy(z).requires_grad_()
    y = torch.nn.functional.silu(t)
    y.sum().backward()
    assert np.allclose(O.activation_fwd("silu", z, 1.0, 1.0), y.detach().numpy(), rtol=1e-13) and np.allclose(O.activation_bwd("silu", z, np.ones_like(z), 1.0, 1.0), t.grad.numpy(), rtol=1e-12)


@pytest.mark.parametrize("fn", FNS)
def test_gradients_are_finite_differences(fn):
    b, m, f, n = 3, 4, 5, 6
    X, Wg, Wu, W2, G = (RNG.standard_normal(s) for s in ((b, m), (m, f), (m, f), (f, n), (b, n)))
    A, h, u = O.gated_fwd(fn, X, Wg, Wu, 0.5, 0.75, 1.0)
    assert np.allclose(A, FNS[fn][0](0.75 * 0.5 * X @ Wg) * (0.5 * X @ Wu), rtol=1e-12)
    loss = lambda h_, u_: (G * ((FNS[fn][0](0.75 * h_) * u_) @ W2)).sum()
    dH, dU = O.gated_bwd(fn, G, W2, 1.0, h, u, 0.75, 1.0, 1.0)
    e = 1e-6
    for i in range(b):
        for j in range(f):
            d = np.zeros((b, f))
            d[i, j] = e
            assert abs((loss(h + d, u) - loss(h - d, u)) / (2 * e) - dH[i, j]) < 1e-7 and abs((loss(h, u + d) - loss(h, u - d)) / (2 * e) - dU[i, j]) < 1e-7
    two = O.gated_bwd(fn, G, W2, 1.0, h, u, 0.75, 2.0, 3.0)
    assert np.allclose(two[0], 2 * dH) and np.allclose(two[1], 3 * dU)


@pytest.mark.parametrize("fn", FNS)
def test_factors_give_unit_scale(fn):
    a, bh, bu = S.gated_scales(*FNS[fn])
    h, u, d = (RNG.standard_normal(400_000) for _ in range(3))
    f, df = FNS[fn]
    assert abs((a * f(h) * u).std() - 1) < 0.02 and abs((bu * f(h) * d).std() - 1) < 0.02 and abs((bh * df(h) * u * d).std() - 1) < 0.02


def test_host_helpers():
    from paper_2303_11257_b200 import lib as L
    for fn, (f, df) in FNS.items():
        for constrained in (False, True):
            assert np.allclose(L.us_scales_gated(fn, constrained), S.gated_scales(f, df, constrained), rtol=1e-6)
    assert np.allclose(L.us_scales_activation("silu"), S.silu_scales(), rtol=1e-6)
    for bad in (5, -1):
        with pytest.raises(L.UnitScaleError):
            L.us_scales_gated(bad)
        with pytest.raises(L.UnitScaleError):
            L.us_scales_activation(bad)


@pytest.mark.parametrize("gate", ["silu", "gelu"])
def test_block_gradients_are_finite_differences_times_constants(gate):
    """Weight gradients of the block without roundings: the true gradients of sum(G R) times the ratio of the factors."""
    T, d, f = 5, 4, 6
    X, W1, W2, G = (RNG.standard_normal(s) for s in ((T, d), (d, 2 * f), (f, d), (T, d)))
    run = lambda W1_, W2_: O.gated_ffn_block(X, W1_, W2_, G, gate, operand="f64", kept="f64", io_dtype="f64")
    r, loss = run(W1, W2), lambda W1_, W2_: (G * run(W1_, W2_).R).sum()
    a, bh, bu = S.gated_scales(*FNS[gate])
    c, e = 0.5 ** 0.5, 1e-5
    up = (T ** -0.5 * d ** -0.5) / (d ** -0.5 * a * c * f ** -0.5)              # of dW1, but for its beta_h or beta_u
    for i in range(d):
        for j in range(2 * f):
            E = np.zeros_like(W1)
            E[i, j] = e
            true = (loss(W1 + E, W2) - loss(W1 - E, W2)) / (2 * e)
            assert abs(true * up * (bh if j < f else bu) - r.dW1[i, j]) < 1e-6
    for i in range(f):
        for j in range(d):
            E = np.zeros_like(W2)
            E[i, j] = e
            assert abs((loss(W1, W2 + E) - loss(W1, W2 - E)) / (2 * e) * T ** -0.5 / (c * f ** -0.5) - r.dW2[i, j]) < 1e-6
