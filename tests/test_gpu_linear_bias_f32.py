"""tanh and sigmoid into float32 of linear ops with a bias: as exact as without one.

Products of zero, so that the argument is in_scale * bias, exactly.  In half steps of float32, u = 2^-24: e^-|z| = 2^(-|z| log2 e) errs by 4 (ex2.approx: 2^-22) and, as the constant and the product are
rounded, by 2 |z| log2 e ln 2 = 2 |z|; it is a part e / (1 + e) of the sum, whose rounding, the division's and the factor's are 1 each; a negative argument's e * r adds 1 and has all of e's error.
So sigmoid is off by (3 + (4 + 2 |z|) e / (1 + e)) u of itself for z >= 0 and (8 + 2 |z|) u for z < 0.  Tanh from 1/8 on is 2 s - 1 with s = sigmoid(2 z): twice the absolute error of s without the factor's
rounding, and one each of its own for the difference and the factor."""
import pytest
import torch

from tests import util as U
from tests.test_gpu_linear_narrow import PAD

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


def _sigmoid_tol(z):
    e = torch.exp(-z.abs())
    s = torch.sigmoid(z)
    return torch.where(z >= 0, 2 + (4 + 2 * z.abs()) * e / (1 + e), 7 + 2 * z.abs()) * u * s


@pytest.mark.parametrize("rows,n", [(3, 4097), (300, 2049)])
@pytest.mark.parametrize("act", ["tanh", "sigmoid"])
@pytest.mark.parametrize("skip", [False, True])
def test_errors(rows, n, act, skip):
    from paper_2303_11257_b200 import lib as L
    gen = torch.Generator().manual_seed(rows)
    z = torch.cat([torch.randn(n // 2, generator=gen), torch.linspace(-60, 60, n - n // 2)]).cuda()
    X, W = torch.zeros((rows, 64), device="cuda").bfloat16(), torch.zeros((64, PAD(n)), device="cuda").bfloat16()[:, :n]
    Y, S = U.empty(rows, n, "f32", PAD(n)), torch.zeros((rows, PAD(n)), device="cuda")[:, :n]
    ep = L.epilogue(act=L.US_ACT_TANH if act == "tanh" else L.US_ACT_SIGMOID, act_in_scale=0.5, act_out_scale=1.5, skip=S if skip else None, skip_coef=0.5 if skip else 0.0, out_coef=1.0)
    L.us_linear_fwd_bias(X, W, 1.0, 2.0 * z, Y, L.new_workspace(), ep)
    d = z.double()
    if act == "sigmoid":
        ref, tol = 1.5 * torch.sigmoid(d), 1.5 * (_sigmoid_tol(d) + u * torch.sigmoid(d))
    else:
        ref = 1.5 * torch.tanh(d)
        tol = torch.where(d.abs() < 0.125, 2.0 ** -21 * ref.abs(), 1.5 * (2 * _sigmoid_tol(2 * d) + 2 * u * torch.tanh(d).abs()))
    off = (Y.double() - ref).abs()
    assert bool((off <= tol * 1.01).all()), float((off / tol).max())
    # of ordinary arguments: the error as a 2-norm.  Rounded quotients and an e that errs evenly by up to 2^-22.5 make 6.4e-8 and 9.1e-8 of it
    part = slice(0, n // 2)
    rel = float((Y[0].double() - ref)[part].norm() / ref[part].norm())
    assert rel < (6.5e-8 if act == "sigmoid" else 1.1e-7), rel


@pytest.mark.parametrize("shape", [(1, 1024, 4096), (1000, 400, 1040), (2600, 80, 1063), (48, 4096, 1024)])
@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
def test_a_bias_of_zero(shape, fmt):
    """But for the last bit of a quotient, by up to a half of its values (a product e r, the difference of tanh, whose s is at least 1/8 of it, and the factor round once more): 2 steps of
    sigmoid, 2 of the s of tanh, which counts from 1/8 on.  Nearly all of them to the bit."""
    from paper_2303_11257_b200 import lib as L
    b, m, n = shape
    gen = torch.Generator(device="cuda").manual_seed(b)
    make = lambda r, c: U.empty(r, c, fmt, PAD(c)).copy_(torch.randn((r, c), generator=gen, device="cuda"))
    X, W, ws = make(b, m), make(m, n), L.new_workspace()
    for act in (L.US_ACT_SIGMOID, L.US_ACT_TANH):
        Y, Z, z = (U.empty(b, n, "f32", PAD(n)) for _ in range(3))
        ep = L.epilogue(act=act, act_out_scale=1.7)
        L.us_linear_fwd(X, W, m ** -0.5, Y, ws, ep)
        L.us_linear_fwd_bias(X, W, m ** -0.5, torch.zeros(n, device="cuda"), Z, ws, ep)
        L.us_linear_fwd(X, W, m ** -0.5, z, ws)
        same = z.abs() >= (0.125 if act == L.US_ACT_TANH else 0.0)
        step = torch.ldexp(torch.ones_like(Y), torch.frexp(Y)[1] - 24) if act == L.US_ACT_SIGMOID else torch.full_like(Y, 1.7 * 2 * 2.0 ** -24)
        assert bool(((Y - Z).abs() <= 2 * step)[same].all()) and float((Y != Z)[same].float().mean()) < 0.02
