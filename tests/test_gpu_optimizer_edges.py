"""us_adamw at the edges of float32: the smallest eps and gradients that it accepts; us_grad_norm of elements whose squares leave its range."""
import math

import numpy as np
import pytest
import torch

from tests import util as U
from tests.test_gpu_optimizer import _check_norm, _norm, _place

pytestmark = pytest.mark.gpu


def _tensors(n, eight):
    from paper_2303_11257_b200 import lib as L
    state = lambda: torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) if eight else torch.zeros(n, device="cuda")
    scale = lambda: torch.zeros(-(-n // 256), device="cuda") if eight else None
    p, g = torch.randn(n, generator=torch.Generator().manual_seed(n)).cuda(), torch.zeros(n, device="cuda")
    return p, g, L.adamw_tensors([p], [g], [state()], [state()], [scale()], [scale()])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n", [77, 512, 1024])
@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1e-38, 3e-37, 1e-30, 1e-8])
def test_elements_without_gradients_stay(eps, n, eight):
    """0 / (0 + eps) is 0 however small eps is; an element with a gradient beside them is stepped by lr."""
    from paper_2303_11257_b200 import lib as L
    p, g, plan = _tensors(n, eight)
    p[5], g[5] = 0.0, 1.0
    before, step = p.clone(), L.new_adamw_step()
    for t in (1, 2, 3):
        L.us_adamw(plan, step, 0.125, eps=eps)
        rest = torch.ones(n, dtype=torch.bool, device="cuda")
        rest[5] = False
        assert torch.equal(p[rest], before[rest])
        # a step is off by 28 half steps of 2^-24 (the tests of steps against the oracle) and one of p's; states in 8 bits, of which this element is the block's largest and has
        # the code 448, by 6 for the scales and their products: 35 in all, 2.1e-6
        assert abs(float(-p[5]) / (0.125 * t) - 1) <= 2.5e-6


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n", [77, 1024])
@pytest.mark.parametrize("g0,tol", [(1e-16, 2.5e-6), (1e-18, 1e-5), (1e-19, 2e-4), (1e-20, 2e-2)])
def test_small_gradients_are_stepped_by_lr(g0, tol, n, eight):
    """sqrt(v) = 10^-1.5 g0 at the first step.  v holds multiples of 2^-149: it is off by 2^-150 / v at most, its root by half of that: 3.5e-7 at 1e-18, 3.5e-5 at 1e-19, 3.5e-3 at 1e-20, and
    below 1e-9 at 1e-16; beside it the step's own 35 half steps of 2^-24, 2.1e-6 (above)."""
    from paper_2303_11257_b200 import lib as L
    p, g, plan = _tensors(n, eight)
    p.zero_()
    g.fill_(g0)
    step = L.new_adamw_step()
    L.us_adamw(plan, step, 0.125, eps=1e-30)
    assert float((p / -0.125 - 1).abs().max()) <= tol
    L.us_adamw(plan, step, 0.125, eps=1e-30)
    # (states in 8 bits: one magnitude, the block's largest, has the code 448, and the scale that brings it back)
    assert float((p / -0.25 - 1).abs().max()) <= tol


def test_a_learning_rate_beyond_float32_is_refused():
    from paper_2303_11257_b200 import lib as L
    p, g, plan = _tensors(77, False)
    before, step = p.clone(), L.new_adamw_step()
    with pytest.raises(L.UnitScaleError):
        L.us_adamw(plan, step, 1e39)
    assert torch.equal(p, before) and step.tolist() == [0, 0]


@pytest.mark.parametrize("fmt,size", [("f32", 1e20), ("bf16", 1e20), ("f32", 3e36), ("f32", 1e-22), ("bf16", 1e-30), ("f32", 1e-38), ("f32", 1e-42), ("fp16", 6e-8), ("fp16", 6e4)])
@pytest.mark.parametrize("shape,pad,shift", [((1, 3), 0, 0), ((1, 1024), 0, 0), ((5, 1031), 0, 0), ((7, 333), 5, 0), ((64, 256), 0, 3)])
def test_norms_of_large_and_small_gradients(shape, pad, shift, fmt, size):
    x = size * np.random.default_rng(5).uniform(0.5, 1.0, shape)
    t, _ = _place(x, fmt, pad, shift)
    wide = U.host_values(t)
    want = math.sqrt(float((wide ** 2).sum()))
    most = float(np.float32(1e-3 * want if want > 1e-38 else 1.0))      # (a float32 of the call)
    n, f = _norm([t], most)
    # (as the other norms; one below 2^-126 is a multiple of 2^-149)
    assert abs(n - want) <= 6 * 2.0 ** -24 * want + 2.0 ** -150
    assert abs(f - min(1.0, most / want)) <= 2.0 ** -24 * min(1.0, most / want) * 1.01


def test_large_beside_small_and_norms_beyond_float32():
    one, tiny, huge = (torch.full((4096,), v, device="cuda") for v in (1.0, 1e-30, 1e25))
    for ts in ([one, tiny], [huge, one, tiny], [tiny, tiny[:77], huge[:5]]):
        _check_norm([U.host_values(t.view(1, -1)) for t in ts], ts, 2.0)
    n, f = _norm([torch.full((1024,), 3e38, device="cuda")])       # 9.6e39
    assert n == math.inf and math.isnan(f)
