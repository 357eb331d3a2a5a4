"""Pins of the oracle's AdamW step, block codes, gradient norm and bias ops: the library optimiser in float64, differences, and values known by hand."""
import math

import numpy as np
import pytest
import torch

from oracle import ops as O


@pytest.mark.parametrize("decay,eps,betas", [(0.0, 1e-8, (0.9, 0.999)), (0.1, 1e-6, (0.5, 0.9)), (0.01, 1e-3, (0.0, 0.99))])
def test_adamw_steps_are_the_library_optimisers(decay, eps, betas):
    rng = np.random.default_rng(0)
    p = rng.standard_normal(50)
    q = torch.nn.Parameter(torch.from_numpy(p.copy()))
    opt = torch.optim.AdamW([q], lr=0.02, betas=betas, eps=eps, weight_decay=decay)
    m = v = np.zeros(50)
    for t in range(1, 8):
        g = rng.standard_normal(50) * 10.0 ** rng.uniform(-4, 2, 50)
        q.grad = torch.from_numpy(3.0 * g)
        opt.step()
        s = O.adamw_step(p, g, m, v, t, 0.02, betas, eps, decay, factor=3.0)
        p, m, v = s.p, s.m, s.v
        assert np.allclose(p, q.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_first_step_is_the_sign_of_the_gradient():
    s = O.adamw_step([1.0, 2.0, 3.0], [4.0, -1e-3, 0.0], np.zeros(3), np.zeros(3), 1, 0.5, eps=1e-12)
    assert np.allclose(s.p, [0.5, 2.5, 3.0], atol=1e-8)


def test_block_codes():
    x = np.zeros(600)
    x[:256] = np.linspace(0, 448, 256)
    x[256:512] = 1e-35                                           # below 2^-100: zeros
    x[512], x[513], x[599] = 2.0, 1e-9, -1.0
    c, s = O.block_codes(x)
    assert s.tolist() == [1.0, 1e-35 / 448, 2.0 / 448] and c[255] == 448.0 and (c[256:512] == 0).all()
    assert c[512] == 448.0 and c[513] == 0.0 and c[599] == -224.0
    assert np.all(np.abs(c[:256] - x[:256]) <= np.maximum(x[:256] * 2.0 ** -4, 2.0 ** -10))
    c, _ = O.block_codes(np.abs(x), positive=True)
    assert c[513] == 2.0 ** -9 and c[514] == 0.0


def test_norm():
    assert O.grad_norm([np.array([3.0]), np.array([[4.0]])], 1.0) == (5.0, 0.2)
    assert O.grad_norm([np.array([3.0]), np.array([[4.0]])], 6.0) == (5.0, 1.0) and O.grad_norm([np.zeros(3)], 1.0) == (0.0, 1.0)
    n, f = O.grad_norm([np.array([math.inf])], 1.0)
    assert n == math.inf and math.isnan(f)


def test_bias_gradient_against_differences():
    rng = np.random.default_rng(1)
    X, W, b, G = rng.standard_normal((6, 4)), rng.standard_normal((4, 3)), rng.standard_normal(3), rng.standard_normal((6, 3))
    loss = lambda b: float((O.linear_bias_fwd(X, W, 0.5, b) * G).sum())
    d = [(loss(b + e) - loss(b - e)) / 2e-5 for e in 1e-5 * np.eye(3)]
    assert np.allclose(d, O.bias_grad(G, 1.0), rtol=1e-8) and np.allclose(O.bias_grad(G, 0.25), 0.25 * G.sum(0))
    # with a unit-normal gradient of b rows, b^-1/2 makes a unit-normal gradient of the bias
    G = rng.standard_normal((4096, 512))
    assert abs(O.bias_grad(G, 4096 ** -0.5).std() - 1) < 0.1


def test_block_with_biases_against_differences():
    """Nothing rounded: both bias gradients are the loss's true ones times constants (a bias is a cut-edge), with L = sum(R * G)."""
    rng = np.random.default_rng(2)
    T, d, f = 7, 5, 6
    X, W1, W2, G = (rng.standard_normal(s) for s in ((T, d), (d, f), (f, d), (T, d)))
    b1, b2 = rng.standard_normal(f), rng.standard_normal(d)
    sc = O.FFNScales.unconstrained(T, d, f)
    run = lambda b1, b2: O.bias_ffn_block(X, W1, b1, W2, b2, G, sc, "f64", "f64", "f64")
    loss = lambda b1, b2: float((run(b1, b2)[0].R * G).sum())
    _, db1, db2 = run(b1, b2)
    h = 1e-5
    d1 = [(loss(b1 + e, b2) - loss(b1 - e, b2)) / (2 * h) for e in h * np.eye(f)]
    d2 = [(loss(b1, b2 + e) - loss(b1, b2 - e)) / (2 * h) for e in h * np.eye(d)]
    branch = math.sqrt(sc.tau)
    assert np.allclose(d2, db2 * branch / sc.beta_w, rtol=1e-6)
    assert np.allclose(d1, db1 * branch / sc.beta_w * (np.float32(sc.alpha2) / np.float32(sc.beta_x2)) * (np.float32(sc.alpha_g) / np.float32(sc.beta_g)), rtol=1e-5)
    plain = O.ffn_block(X, W1, W2, G, sc, operand="f64", h_dtype="f64", io_dtype="f64")
    zero, _, _ = O.bias_ffn_block(X, W1, np.zeros(f), W2, np.zeros(d), G, sc, "f64", "f64", "f64")
    assert np.allclose(plain.R, zero.R) and np.allclose(plain.dW1, zero.dW1, atol=1e-6) and np.allclose(plain.dX, zero.dX)
