"""us_adamw and us_grad_norm against the oracle.

Tolerances in units of u = 2^-24, half a float32 step.  m: the factors beta and 1 - beta are rounded (1 each), so are grad_factor * grad,
its product and the sum: at most 5 of beta |m| + (1 - beta) |g|.  v (all terms positive): 7, taken as 8; its root 4, and 2 for the approximate root: 6.
1 - beta^t: the exponent t log(beta) holds 3 roundings, which move 1 - e^z by no more than themselves, expm1 2: 5; its root and reciprocal
4.5; denominator 6 + 4.5 + 2 roundings, taken as 13; the division is off by up to 2 steps, 4; rate: lr, 1 - beta1^t, a division and
two factors: 10.  So the gradient's part of the step is off by 13 + 4 + 10 + 1 = 28 of itself and 5 of rate (beta |m| + (1 - beta) |g|) / denominator; the
decayed part by 5 of itself; their sum and p are rounded once each: 1 of p, 1 of the sum (in the 28 and 5, taken as 30 and 6).
Codes: half a step of E4M3 (2^-4 of the value, 2^-10 of the scale below the smallest normal number) beside those; for a positive value the
smallest code is 2^-9 of the scale.  Norm: 8 squares are added in float32, 8 of the sum, 4 of its root, and 1 to store it."""
import math

import numpy as np
import pytest
import torch

from oracle import formats as F
from oracle import ops as O
from tests import util as U

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


def _lib():
    from paper_2303_11257_b200 import lib
    return lib


def _place(x, fmt, pad=0, shift=0):
    """x on the device with `pad` more columns a row (NaN) and `shift` elements behind a 16-byte boundary; and all of that memory."""
    rows, cols = x.shape
    dt = U.TORCH_OF[fmt]
    one = torch.full((rows * (cols + pad) + shift + 16,), math.nan, dtype=torch.float32).to(dt).cuda()
    t = one[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(np.float32(x)).cuda().to(dt))
    return t, one


class Case:
    """A tensor of a call: on the device, and the oracle's state of it."""

    def __init__(self, rows, cols, eight=False, grad="f32", copy=None, pads=(0, 0, 0), shifts=(0, 0, 0, 0, 0), decay=0.0, lr_factor=1.0, copy_scale=1.0, fresh=False, seed=0):
        rng = np.random.default_rng(seed + 131 * rows + cols)
        n = rows * cols
        self.eight, self.grad_fmt, self.copy_fmt, self.decay, self.lr_factor, self.copy_scale = eight, grad, copy, decay, lr_factor, copy_scale
        sigma = np.exp(rng.standard_normal((rows, cols)))
        self.p = np.float32(rng.standard_normal((rows, cols)))
        g = np.float32(sigma * rng.standard_normal((rows, cols)))
        self.dev_p, self.all_p = _place(self.p, "f32", pads[0], shifts[0])
        self.dev_g, _ = _place(g, grad, pads[1], shifts[1])
        self.g = U.host_values(self.dev_g)
        m = np.zeros(n) if fresh else (0.3 * sigma * rng.standard_normal((rows, cols))).ravel()
        root = np.zeros(n) if fresh else sigma.ravel()
        if eight:
            (cm, sm), (cv, sv) = O.block_codes(m), O.block_codes(root, positive=True)
            self.scales = [torch.from_numpy(np.float32(s)).cuda() for s in (sm, sv)]
            self.state = [_place(c.reshape(1, n), "e4m3", 0, s)[0] for c, s in ((cm, shifts[2]), (cv, shifts[3]))]
        else:
            self.scales = [None, None]
            self.state = [_place(np.float32(x).reshape(1, n), "f32", 0, s)[0] for x, s in ((m, shifts[2]), (root ** 2, shifts[3]))]
        self.copy, self.all_copy = (None, None) if copy is None else _place(np.zeros((rows, cols)), copy, pads[2], shifts[4])
        self.pads, self.shifts, self.shape = pads, shifts, (rows, cols)

    def held(self):
        """m and v as they are held."""
        a, b = (U.host_values(t).ravel() for t in self.state)
        if not self.eight:
            return a, b
        sm, sv = (np.repeat(s.double().cpu().numpy(), 256)[:a.size] for s in self.scales)
        return sm * a, (sv * b) ** 2

    def check(self, before, t, lr, betas=(0.9, 0.999), eps=1e-8, factor=1.0, what=""):
        """The state after step t against the oracle's step from `before` = (p, m, v) as they were held."""
        p0, m0, v0 = before
        g = self.g.ravel()
        rate = float(np.float32(lr)) * self.lr_factor
        w = O.adamw_step(p0, g, m0, v0, t, lr * self.lr_factor, betas, eps, self.decay, factor)
        tol_m = 5 * u * (betas[0] * np.abs(m0) + (1 - betas[0]) * np.abs(factor * g))
        tol_p = 1.05 * u * (np.abs(w.p) + 6 * np.abs(w.decayed) + 30 * np.abs(w.update) + rate / (1 - betas[0] ** t) * (tol_m / u) / w.denominator)
        p = U.host_values(self.dev_p).ravel()
        assert (np.abs(p - w.p) <= tol_p).all(), (what, "p", float((np.abs(p - w.p) / tol_p).max()))
        m, v = self.held()
        if self.eight:
            root, got = np.sqrt(w.v), np.sqrt(v)
            for name, x, y, tol, positive in (("m", w.m, m, tol_m, False), ("root of v", root, got, 6 * u * root, True)):
                blocks = -(-x.size // 256)
                pad = np.zeros(256 * blocks)
                pad[:x.size] = np.abs(x)
                most = pad.reshape(blocks, 256).max(1)
                scale = self.scales[positive].double().cpu().numpy()
                assert (np.abs(scale * 448 - most) <= 8 * u * most + (0 if positive else 5 * u * most)).all() or name == "m"
                s = np.repeat(scale, 256)[:x.size]
                half = np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10)
                if positive:
                    half = np.where((x > 0) & (x < s * 2.0 ** -9), s * 2.0 ** -9, half)
                    assert ((y > 0) == (x > 0)).all(), what
                ok = np.abs(y - x) <= half * (1 + 1e-5) + 2 * tol
                assert ok.all(), (what, name, int((~ok).sum()))
        else:
            assert (np.abs(m - w.m) <= tol_m).all() and (np.abs(v - w.v) <= 8 * u * w.v).all(), what
        if self.copy is not None:
            want = U.TORCH_OF[self.copy_fmt]
            y = np.float32(self.copy_scale) * np.float32(p)
            ref = F.quantise(y, F.FORMATS[self.copy_fmt]) if self.copy_fmt != "f32" else y.astype(np.float64)
            assert np.array_equal(U.host_values(self.copy).ravel(), ref), (what, want)
        # what lies between the rows and behind them is as it was
        for whole, t_, pad, shift in ((self.all_p, self.dev_p, self.pads[0], self.shifts[0]),) + (((self.all_copy, self.copy, self.pads[2], self.shifts[4]),) if self.copy is not None else ()):
            rows, cols = self.shape
            h = whole.float().cpu()
            inside = h[shift:shift + rows * (cols + pad)].view(rows, cols + pad)
            assert bool(torch.isnan(inside[:, cols:]).all()) and bool(torch.isnan(h[:shift]).all()) and bool(torch.isnan(h[shift + rows * (cols + pad):]).all()), what


def _plan(cases):
    L = _lib()
    return L.adamw_tensors([c.dev_p for c in cases], [c.dev_g for c in cases], [c.state[0] for c in cases], [c.state[1] for c in cases], [c.scales[0] for c in cases],
                           [c.scales[1] for c in cases], [c.copy for c in cases], [c.copy_scale for c in cases], [c.decay for c in cases], [c.lr_factor for c in cases])


def _before(cases):
    return [(U.host_values(c.dev_p).ravel(),) + c.held() for c in cases]


def _steps(cases, steps=2, lr=0.01, made=0, **kw):
    L = _lib()
    plan, step = _plan(cases), L.new_adamw_step(made)
    for t in range(made + 1, made + 1 + steps):
        before = _before(cases)
        L.us_adamw(plan, step, lr, **kw)
        torch.cuda.synchronize()
        assert step.tolist() == [t, 0]
        checks = {k: v for k, v in kw.items() if k in ("betas", "eps")}
        for k, (c, b) in enumerate(zip(cases, before)):
            c.check(b, t, lr, what=(k, c.shape, t), **checks)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("shape", [(1, 1), (1, 3), (1, 255), (1, 256), (1, 257), (5, 100), (37, 1031), (64, 512), (300, 4)])
def test_sizes(shape, eight):
    _steps([Case(*shape, eight=eight, copy="e4m3", decay=0.1)], steps=3)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("grad,copy", [("f32", None), ("bf16", "bf16"), ("fp16", "fp16"), ("f32", "e5m2"), ("bf16", "f32"), ("fp16", "e4m3")])
def test_types(grad, copy, eight):
    _steps([Case(33, 264, eight=eight, grad=grad, copy=copy, copy_scale=0.5, decay=0.01, lr_factor=0.5)])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("cols", [96, 130, 1031, 260])
@pytest.mark.parametrize("pads", [(0, 0, 4), (0, 4, 0), (4, 0, 0), (8, 12, 16), (1, 3, 5), (0, 0, 7), (2, 0, 0)])
def test_padded_rows(cols, pads, eight):
    """Groups of four that end at a row, that cross it, and matrices with and without padding beside one another."""
    _steps([Case(7, cols, eight=eight, grad="bf16", copy="e4m3", pads=pads, decay=0.1)])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("which", range(5))
@pytest.mark.parametrize("by", [1, 2])
def test_starts_between_boundaries(which, by, eight):
    shifts = tuple(by if i == which else 0 for i in range(5))
    _steps([Case(9, 200, eight=eight, grad="fp16", copy="bf16", shifts=shifts)])


def test_many_tensors_of_all_kinds():
    """More than a launch describes, some without elements."""
    kinds = [dict(), dict(eight=True), dict(eight=True, copy="e4m3"), dict(grad="bf16", copy="bf16", pads=(0, 0, 3)), dict(decay=0.2, lr_factor=0.0), dict(fresh=True)]
    rng = np.random.default_rng(3)
    cases = [Case(int(rng.integers(0, 4)), int(rng.integers(0, 400)), seed=i, **kinds[i % len(kinds)]) for i in range(530)]
    _steps(cases, steps=2)


@pytest.mark.parametrize("count", [1, 30, 31, 240, 241])
def test_tables(count):
    _steps([Case(1, 5 + i, seed=i, fresh=i % 2 == 0) for i in range(count)], steps=1)


@pytest.mark.parametrize("kw", [dict(betas=(0.0, 0.0)), dict(betas=(0.5, 0.9), eps=1e-3), dict(betas=(0.0, 0.999)), dict(lr=0.0), dict(made=1000), dict(made=10 ** 7),
                                dict(made=2 ** 40, steps=1)])
@pytest.mark.parametrize("eight", [False, True])
def test_options(kw, eight):
    _steps([Case(20, 100, eight=eight, decay=0.1, copy="e4m3")], **kw)


def test_factors_in_device_memory():
    L = _lib()
    lr, gf = torch.tensor([0.25], device="cuda"), torch.tensor([9.0, 0.125], device="cuda")
    cases = [Case(20, 100), Case(10, 77, eight=True)]
    step, before = L.new_adamw_step(4), _before(cases)
    L.us_adamw(_plan(cases), step, 0.04, lr_factor=lr, grad_factor=gf[1:])
    for c, b in zip(cases, before):
        c.check(b, 5, 0.01, factor=0.125)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_factor_that_is_not_finite_makes_no_step(bad):
    L = _lib()
    cases = [Case(20, 100, copy="e4m3"), Case(10, 77, eight=True)] + [Case(1, 9, seed=i) for i in range(240)]
    step, plan = L.new_adamw_step(4), _plan(cases)
    before, copies = _before(cases), cases[0].copy.float().clone()
    L.us_adamw(plan, step, 0.04, grad_factor=torch.tensor([bad], device="cuda"))
    assert step.tolist() == [4, 0] and torch.equal(cases[0].copy.float(), copies)
    for b, a in zip(before, _before(cases)):
        assert all(np.array_equal(x, y) for x, y in zip(b, a))
    L.us_adamw(plan, step, 0.04)                                   # and the next one does
    assert step.tolist() == [5, 0]
    for c, b in zip(cases, before):
        c.check(b, 5, 0.04)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_gradients_that_are_not_finite(bad):
    """They spoil their own element, infinite ones the block of states in 8 bits from the next step on."""
    L = _lib()
    a, b = Case(4, 200), Case(4, 200, eight=True)
    for c in (a, b):
        c.dev_g[1, 100] = bad                                      # element 300: block 1
    step, plan, before = L.new_adamw_step(), _plan([a, b]), _before([a, b])
    L.us_adamw(plan, step, 0.01)
    for c, was in zip((a, b), before):
        p = U.host_values(c.dev_p).ravel()
        assert np.isnan(p[300]) and np.isfinite(np.delete(p, 300)).all()
        w = O.adamw_step(was[0], c.g.ravel(), was[1], was[2], 1, 0.01)
        assert np.allclose(np.delete(p, 300), np.delete(w.p, 300), rtol=1e-5, atol=1e-6)
    L.us_adamw(plan, step, 0.01)
    pa, pb = U.host_values(a.dev_p).ravel(), U.host_values(b.dev_p).ravel()
    assert np.isnan(pa[300]) and np.isfinite(np.delete(pa, 300)).all()
    spoilt = slice(300, 301) if math.isnan(bad) else slice(256, 512)
    assert np.isnan(pb[spoilt]).all() and np.isfinite(np.delete(pb, spoilt)).all()


def test_blocks_of_zeros_and_of_far_apart_values():
    """Gradients of zero leave zeros; an element 10^6 below its block's largest keeps a denominator, and a code of m only if it has one."""
    L = _lib()
    c = Case(1, 768, eight=True, fresh=True)
    c.dev_g.zero_()
    c.dev_g[0, 256:512] = 1e-6
    c.dev_g[0, 300] = 10.0
    c.dev_g[0, 512:] = 1e-33
    c.g = U.host_values(c.dev_g)
    step, plan = L.new_adamw_step(), _plan([c])
    for t in (1, 2, 3):
        before = _before([c])[0]
        L.us_adamw(plan, step, 0.01)
        torch.cuda.synchronize()
        p = U.host_values(c.dev_p).ravel()
        assert np.isfinite(p).all() and np.array_equal(p[:256], c.p.ravel()[:256])
        # a step is about lr at most: no element lost its denominator
        assert (np.abs(p - before[0]) <= 0.0101).all()
    assert (c.scales[0][0] == 0) and (c.scales[1][0] == 0) and (U.host_values(c.state[1]).ravel()[256:512] > 0).all()


def test_first_moments_in_8_bits_round_as_the_formula_says():
    """Operation by operation in float32, to the bit: codes and scales of m do not depend on fused forms."""
    L = _lib()
    gen = torch.Generator(device="cuda").manual_seed(11)
    n = 256 * 4000
    normal = lambda: torch.randn(n, generator=gen, device="cuda")
    p, g = normal(), (normal() * torch.exp(normal())).bfloat16()
    m = (normal() * torch.exp(normal())).view(-1, 256)
    sm = m.abs().amax(1) / 448.0
    cm = (m * ((1 / m.abs().amax(1)) * 448.0)[:, None]).to(torch.float8_e4m3fn).flatten()
    cv, sv = torch.ones(n, device="cuda").to(torch.float8_e4m3fn), torch.ones(n // 256, device="cuda")
    factor = torch.tensor([0.7], device="cuda")
    for _ in range(3):
        x = 0.9 * (cm.float().view(-1, 256) * sm[:, None]) + (1 - 0.9) * (g.float() * factor).view(-1, 256)
        most = x.abs().amax(1)
        want_scale, want = most * torch.tensor(1 / 448, device="cuda"), (x * ((1 / most) * 448.0)[:, None]).to(torch.float8_e4m3fn).flatten()
        L.us_adamw(L.adamw_tensors([p], [g], [cm], [cv], [sm], [sv]), L.new_adamw_step(5), 1e-3, grad_factor=factor)
        assert torch.equal(sm, want_scale) and torch.equal(cm.view(torch.uint8), want.view(torch.uint8))


def test_captured_steps_count_on_and_agree():
    L = _lib()
    make = lambda: [Case(20, 100, copy="e4m3", decay=0.1), Case(10, 777, eight=True)] + [Case(1, 9, seed=i) for i in range(250)]
    a, b = make(), make()
    pa, pb, sa, sb = _plan(a), _plan(b), L.new_adamw_step(), L.new_adamw_step()
    for _ in range(4):
        L.us_adamw(pa, sa, 0.01)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.us_adamw(pb, sb, 0.01)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.us_adamw(pb, sb, 0.01)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert sa.tolist() == sb.tolist() == [4, 0]
    for x, y in zip(a, b):
        assert torch.equal(x.dev_p, y.dev_p) and all(torch.equal(s.view(torch.uint8), r.view(torch.uint8)) for s, r in zip(x.state, y.state))


def test_elements_beyond_32_bits():
    """2^32 + 2^17 elements; the last ones and some around 2^31 and 2^32 against the oracle."""
    L = _lib()
    rows, cols = 65538, 65536
    n = rows * cols
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    p = torch.ones((rows, cols), device="cuda")
    g = torch.full((rows, cols), 0.5, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros((rows, cols), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    copy = torch.zeros((rows, cols), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    sm, sv = torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")
    marks = [0, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, 2 ** 32 + 77, n - 1]
    flat = g.view(-1)
    for i, k in enumerate(marks):
        flat[k] = -float(i + 1)
    L.us_adamw(L.adamw_tensors([p], [g], [m], [v], [sm], [sv], [copy]), L.new_adamw_step(), 0.25)
    torch.cuda.synchronize()
    want = torch.full((), 0.75, device="cuda")
    for i, k in enumerate(marks):
        assert abs(float(p.view(-1)[k]) - 1.25) < 1e-5 and float(copy.view(-1)[k]) == 1.25
        most = max(j + 1 for j, other in enumerate(marks) if other // 256 == k // 256)      # (two marks share a block)
        assert abs(float(sm[k // 256]) * 448 - 0.1 * most) < 1e-5 * most
    for chunk in p.view(-1).split(1 << 30):
        assert int(((chunk - want).abs() > 1e-5).sum()) <= 7
    assert int(sum(((c - want).abs() > 1e-5).sum() for c in p.view(-1).split(1 << 30))) == 7


# ------------------------------------------------------------ norm

def _norm(tensors, most=1.0, ws=None):
    L = _lib()
    out = torch.full((2,), -1.0, device="cuda")
    ws = torch.zeros(L.us_grad_norm_workspace_bytes(), dtype=torch.uint8, device="cuda") if ws is None else ws
    L.us_grad_norm(tensors, most, out, ws)
    return [float(x) for x in out.double()]


def _check_norm(arrays, tensors, most=1.0, ws=None):
    n, f = _norm(tensors, most, ws)
    wn, wf = O.grad_norm(arrays, most)
    assert abs(n - wn) <= 6 * u * wn and abs(f - wf) <= 7 * u * wf, (n, wn, f, wf)


@pytest.mark.parametrize("fmt", ["f32", "bf16", "fp16"])
@pytest.mark.parametrize("shape,pad,shift", [((1, 1), 0, 0), ((1, 1023), 0, 0), ((1, 1024), 0, 1), ((3, 1025), 0, 0), ((7, 333), 5, 0), ((64, 256), 8, 0), ((64, 256), 0, 3), ((500, 2096), 80, 0)])
def test_norm(shape, pad, shift, fmt):
    x = np.random.default_rng(5).standard_normal(shape)
    t, _ = _place(x, fmt, pad, shift)
    _check_norm([U.host_values(t)], [t])


@pytest.mark.parametrize("count", [2, 80, 81, 640, 641, 1500])
def test_norm_of_many(count):
    rng = np.random.default_rng(count)
    ts = [_place(rng.standard_normal((int(rng.integers(0, 3)), int(rng.integers(0, 300)))) * 10.0 ** rng.uniform(-3, 3), ["f32", "bf16", "fp16"][i % 2])[0] for i in range(count)]
    L = _lib()
    ws = torch.zeros(L.us_grad_norm_workspace_bytes(), dtype=torch.uint8, device="cuda")
    for _ in range(2):                                             # the workspace is ready for the next call
        _check_norm([U.host_values(t) for t in ts], ts, 1e3, ws)


def test_norms_at_the_edges():
    z = torch.zeros(10, device="cuda")
    assert _norm([z]) == [0.0, 1.0] and _norm([z[:0]]) == [0.0, 1.0] and _norm([z + 1], 100.0)[1] == 1.0 and _norm([z + 1e9], math.inf)[1] == 1.0
    for bad in (math.nan, math.inf):
        x = torch.ones(5000, device="cuda")
        x[4321] = bad
        n, f = _norm([z, x])
        assert not math.isfinite(n) and math.isnan(f)
    x = torch.full((3000,), 1e15, device="cuda")                   # squares of 1e30
    assert abs(_norm([x])[0] / (1e15 * math.sqrt(3000)) - 1) < 1e-6


def test_norm_of_a_long_tensor_is_repeatable():
    x = torch.randn(1 << 26, device="cuda")
    a = _norm([x, x[:12345]])
    assert all(_norm([x, x[:12345]]) == a for _ in range(3))
    want = math.sqrt(float(x.double().square().sum()) + float(x[:12345].double().square().sum()))
    assert abs(a[0] - want) <= 6 * u * want


def test_clipped_steps_captured_together():
    """Norm and step of a training loop as one captured graph, the factor handed over in device memory."""
    L = _lib()
    c = Case(40, 300)
    c2 = Case(1, 300, eight=True)
    plan, step = _plan([c, c2]), L.new_adamw_step()
    grads, out = L.mats([c.dev_g, c2.dev_g]), torch.zeros(2, device="cuda")
    ws = torch.zeros(L.us_grad_norm_workspace_bytes(), dtype=torch.uint8, device="cuda")

    def go():
        L.us_grad_norm(grads, 2.0, out, ws)
        L.us_adamw(plan, step, 0.01, grad_factor=out[1:])
    before = _before([c, c2])
    go()
    _, factor = O.grad_norm([c.g, c2.g], 2.0)
    for x, b in zip((c, c2), before):
        x.check(b, 1, 0.01, factor=float(out[1].double()))
    assert abs(float(out[1]) - factor) <= 1e-6 * factor
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    c.dev_g[0, 0] = math.nan
    g.replay()
    assert step.tolist() == [1, 0]
    c.dev_g[0, 0] = 1.0
    g.replay()
    assert step.tolist() == [2, 0]
