"""us_adamw with states in 8 bits that are rounded randomly: codes against the oracle's, the paths of a launch against one another, and many steps against states in 32 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import ops as O
from tests import util as U
from tests.test_gpu_optimizer import Case

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


def _lib():
    from paper_2303_11257_b200 import lib
    return lib


def _plan(cases, rounding=1):
    L = _lib()
    return L.adamw_tensors([c.dev_p for c in cases], [c.dev_g for c in cases], [c.state[0] for c in cases], [c.state[1] for c in cases], [c.scales[0] for c in cases],
                           [c.scales[1] for c in cases], [c.copy for c in cases], [c.copy_scale for c in cases], [c.decay for c in cases], [c.lr_factor for c in cases], rounding=rounding)


def _check_codes(c, before, t, what, betas=(0.9, 0.999)):
    """Codes are the oracle's, except where the way behind a value and its fraction are 1 together up to the rounding of the value: m's by the 5 half steps of its terms, both by 10 more of themselves
    for scale, reciprocal and root, of up to 16 code steps; 2^-21 of a step where 2^-6 is added."""
    p0, m0, v0 = before
    g = c.g.ravel()
    w = O.adamw_step(p0, g, m0, v0, t, 0.0, betas)
    for x, state, scale, fractions, positive, off in ((w.m, c.state[0], c.scales[0], O.rounding_bits(t, g.size)[0], False, 5 * u * (betas[0] * np.abs(m0) + (1 - betas[0]) * np.abs(g))),
                                                      (np.sqrt(w.v), c.state[1], c.scales[1], O.rounding_bits(t, g.size)[1], True, 0.0)):
        codes, scales = O.block_codes(x, positive=positive, fractions=fractions)
        got, s = U.host_values(state).ravel(), scale.double().cpu().numpy()
        blocks = np.array([np.broadcast_to(off, x.shape)[i:i + 256].max() for i in range(0, x.size, 256)])
        assert (np.abs(s - scales) <= 10 * u * scales + blocks / 448).all(), what
        each = np.repeat(scales, 256)[:x.size]
        value = np.abs(x) / np.where(each > 0, each, 1.0)
        if positive:
            value = np.where(value > 0, np.maximum(value, 2.0 ** -9), value)
        apart = 2.0 ** (np.floor(np.log2(np.maximum(value, 2.0 ** -6))) - 3)
        way = value / apart + fractions
        tol = 16 * 10 * u + 2.0 ** -21 + np.where(each > 0, off / np.where(each > 0, each, 1.0), 0.0) / apart
        edge = np.abs(way - np.round(way)) <= tol
        edge |= np.abs(value - 2.0 ** np.round(np.log2(np.maximum(value, 2.0 ** -9)))) <= tol * apart       # (where the steps change)
        assert edge.mean() <= 0.02 + 3 / x.size
        assert np.array_equal(got[~edge], codes[~edge]), (what, positive, int((got != codes).sum()))
        assert (np.abs(got - np.sign(x) * np.minimum(value, 448.0)) <= apart * (1 + tol)).all()


def _steps(cases, steps=2, made=0):
    L = _lib()
    plan, step = _plan(cases), L.new_adamw_step(made)
    for t in range(made + 1, made + 1 + steps):
        before = [(U.host_values(c.dev_p).ravel(),) + c.held() for c in cases]
        L.us_adamw(plan, step, 0.01)
        torch.cuda.synchronize()
        assert step.tolist() == [t, 0]
        for k, (c, b) in enumerate(zip(cases, before)):
            _check_codes(c, b, t, (k, c.shape, t))


@pytest.mark.parametrize("shape", [(1, 1), (1, 3), (1, 255), (1, 256), (1, 257), (5, 100), (37, 1031), (64, 512), (300, 4)])
def test_codes(shape):
    _steps([Case(*shape, eight=True, copy="e4m3", decay=0.1)], steps=3)


@pytest.mark.parametrize("grad", ["f32", "bf16", "fp16"])
@pytest.mark.parametrize("made", [0, 999, 2 ** 32 + 5])
def test_codes_of_late_steps_and_other_gradients(grad, made):
    _steps([Case(33, 264, eight=True, grad=grad, fresh=made == 0)], made=made)


def test_every_path_rounds_alike():
    """Dense, padded and unaligned tensors, alone and among others: the same states, to the bit."""
    L = _lib()
    kinds = [dict(), dict(pads=(4, 0, 0)), dict(pads=(0, 3, 0)), dict(shifts=(1, 0, 0, 0, 0)), dict(shifts=(0, 0, 1, 0, 0)), dict(shifts=(0, 0, 0, 2, 0)), dict(copy="bf16", pads=(0, 0, 7))]
    cases = [Case(40, 129, eight=True, **k) for k in kinds]
    others = [Case(40, 129), Case(40, 129, eight=True), Case(3, 5, eight=True)] + [Case(1, 300, eight=True, seed=i) for i in range(240)]
    alone = Case(40, 129, eight=True)
    a, b = L.new_adamw_step(), L.new_adamw_step()
    plan = _plan(cases + others, [1] * len(cases) + [0, 0, 1] + [1] * 240)
    for t in range(3):
        L.us_adamw(plan, a, 0.01)
        L.us_adamw(_plan([alone]), b, 0.01)
    assert a.tolist() == b.tolist() == [3, 0]
    for c in cases:
        assert all(torch.equal(x.reshape(-1).view(torch.uint8), y.reshape(-1).view(torch.uint8)) for x, y in zip(c.state + c.scales, alone.state + alone.scales))
        assert torch.equal(c.dev_p, alone.dev_p)
    nearest = Case(40, 129, eight=True)
    step = L.new_adamw_step()
    for t in range(3):
        L.us_adamw(_plan([nearest], 0), step, 0.01)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(nearest.state, others[1].state))
    assert not torch.equal(nearest.state[1].view(torch.uint8), alone.state[1].view(torch.uint8))


def test_captured_steps_round_as_others_do():
    L = _lib()
    a, b = Case(20, 777, eight=True), Case(20, 777, eight=True)
    pa, pb, sa, sb = _plan([a]), _plan([b]), L.new_adamw_step(), L.new_adamw_step()
    for _ in range(4):
        L.us_adamw(pa, sa, 0.01)
    L.us_adamw(pb, sb, 0.01)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.us_adamw(pb, sb, 0.01)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert sa.tolist() == sb.tolist() == [4, 0] and torch.equal(a.dev_p, b.dev_p)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a.state, b.state))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_gradients_that_are_not_finite(bad):
    L = _lib()
    c = Case(4, 200, eight=True)
    c.dev_g[1, 100] = bad                                          # element 300: block 1
    step, plan = L.new_adamw_step(), _plan([c])
    L.us_adamw(plan, step, 0.01)
    p = U.host_values(c.dev_p).ravel()
    assert np.isnan(p[300]) and np.isfinite(np.delete(p, 300)).all()
    if math.isnan(bad):
        assert bool(c.state[0].float().view(-1)[300].isnan()) and bool(c.state[1].float().view(-1)[300].isnan())
    L.us_adamw(plan, step, 0.01)
    p = U.host_values(c.dev_p).ravel()
    spoilt = slice(300, 301) if math.isnan(bad) else slice(256, 512)
    assert np.isnan(p[spoilt]).all() and np.isfinite(np.delete(p, spoilt)).all()


def _run(fall, states, steps, falls, last, n=1 << 14, **kw):
    """(root of v, mean size of the last steps) of every element; gradients are the same for all kinds of states."""
    from paper_2303_11257_b200 import optim
    gen = torch.Generator(device="cuda").manual_seed(3)
    sigma = torch.exp(torch.randn(n, generator=gen, device="cuda"))
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    opt, size = optim.AdamW([p], [g], lr=1e-3, weight_decay=0.0, states=states, **kw), torch.zeros(n, device="cuda")
    for t in range(steps):
        torch.randn(n, generator=gen, device="cuda", out=g)
        g.mul_(sigma)
        if t == falls:
            sigma[::2] *= fall
        p.zero_()                                                  # (p is then the step)
        opt.step()
        if t >= steps - last:
            size += p.abs() / last
    if states == "32bit":
        return opt.v[0].sqrt().double(), size.double()
    return (opt.v[0].float().view(-1, 256) * opt.v_scale[0][:, None]).flatten().double(), size.double()


@pytest.mark.parametrize("fall", [0.1, 0.0])
def test_many_steps_follow_states_in_32_bits(fall):
    """Gradients of log-normal size; after 1000 of 6000 steps those of every second element fall.  sqrt(v) keeps the mean, and steps the size, that they have with states in 32 bits.

    A step changes sqrt(v) by up to 0.05 % of itself, so one of about 180 goes to another code, 9 % away: the square of the spread grows by 4.5e-5 a step.  Where gradients keep their size it
    is forgotten at the rate 0.002 and stays at 0.0225: spread 0.15, sqrt(v) 1.1 % larger in the mean, 1 / sqrt(v) 2.3 %; means of 8192 are off by 0.15 / 90, four of them 0.007: 0.02 and 0.03.  Where they have
    fallen nothing is forgotten for up to 5000 steps: 0.225; a mean of 8192 numbers spread by 0.5 is off by 0.0055, four of them 0.022, taken as 0.03 (that of a product of many factors has a longer
    tail), and 1 / sqrt(v) is up to 1.25 times as large in the mean; 0.28 with the error."""
    root, size = _run(fall, "32bit", 6000, 1000, 200)
    r, s = _run(fall, "8bit", 6000, 1000, 200, rounding="random")
    for part, tol_root, tol_step in ((slice(0, None, 2), 0.03, 0.28), (slice(1, None, 2), 0.02, 0.03)):
        assert abs(float((r[part] / root[part]).mean()) - 1) < tol_root
        assert abs(float(s[part].mean() - size[part].mean())) <= tol_step * float(size[part].mean()) + 1e-12
    assert fall or float(s[::2].max()) == 0.0                      # the first moments of elements without gradients have come to zero


def test_the_driver_hands_the_rounding_on():
    from paper_2303_11257_b200 import optim
    p = [torch.randn(30, 50, device="cuda"), torch.randn(77, device="cuda")]
    g = [torch.randn(30, 50, device="cuda"), torch.randn(77, device="cuda")]
    a, b = (optim.AdamW([t.clone() for t in p], g, states="8bit", rounding=r) for r in ("random", "nearest"))
    for _ in range(2):
        a.step(), b.step()
    assert not torch.equal(a.v[0].view(torch.uint8), b.v[0].view(torch.uint8))
    c = optim.AdamW([t.clone() for t in a.params], g, states="8bit", rounding="random")
    c.load_state_dict(a.state_dict())
    a.step(), c.step()
    assert all(torch.equal(x, y) for x, y in zip(a.params + a.v_scale, c.params + c.v_scale)) and all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a.v, c.v))
