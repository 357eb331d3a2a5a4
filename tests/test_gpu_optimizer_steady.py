"""us_adamw over many more units than the CTAs of a launch begin with: chunks that CTAs take from the counter, and units fetched ahead across the ends of tensors and between whole units and others.
Every element against the oracle, with the tolerances of the tests of steps, and the scales of every block of states in 8 bits, of m too."""
import numpy as np
import pytest
import torch

from oracle import ops as O
from tests import util as U
from tests.test_gpu_adamw_rounding import _check_codes
from tests.test_gpu_optimizer import Case, u

pytestmark = pytest.mark.gpu

# what tensors look like: dense (all accesses in pieces), with padded rows, with starts between boundaries, with copies of every kind of place
KINDS = [dict(copy="e4m3"), dict(grad="bf16", copy="bf16"), dict(grad="bf16"), dict(pads=(4, 0, 0)), dict(grad="fp16", copy="e5m2", pads=(0, 0, 16)), dict(copy="fp16", pads=(0, 0, 7)),
         dict(grad="fp16", shifts=(0, 2, 0, 0, 0)), dict(shifts=(0, 0, 1, 0, 0)), dict(copy="f32", shifts=(0, 0, 0, 4, 0)), dict(grad="bf16", copy="e4m3", fresh=True, decay=0.1)]


def _cases(tensors, elements, eight, seed):
    """`tensors` of them, elements in all, of sizes that differ by a factor of ten and are no multiples of anything; among them some of whole units and some small ones."""
    rng = np.random.default_rng(seed)
    cases = []
    for i in range(tensors):
        n = int(elements / tensors * 10 ** rng.uniform(-0.6, 0.4))
        cols = int(rng.choice([4, 63, 130, 256, 520, 1031, 2048]))
        shape = (1, int(rng.integers(1, 700))) if i % 7 == 3 else (1, max(1, n // 512) * 512) if i % 7 == 5 else (max(1, n // cols), cols)
        cases.append(Case(*shape, eight=eight, seed=i, **KINDS[(i + i // 10) % len(KINDS)]))
    return cases


def _check_scales(c, before, what):
    """Scales are the oracle's largest magnitudes / 448: off by what the largest of a block's values can be (m: 5 half steps of its terms; roots: 6), and 3 for 1 / 448 and the product."""
    p0, m0, v0 = before
    g, at = c.g.ravel(), np.arange(0, m0.size, 256)
    w = O.adamw_step(p0, g, m0, v0, 1, 0.0)
    for x, off, scale in ((np.abs(w.m), 5 * u * (0.9 * np.abs(m0) + 0.1 * np.abs(g)), c.scales[0]), (np.sqrt(w.v), 6 * u * np.sqrt(w.v), c.scales[1])):
        most = np.maximum.reduceat(x, at)
        assert (np.abs(448 * scale.double().cpu().numpy() - most) <= np.maximum.reduceat(off, at) + 3 * u * most).all(), what


# (elements that CTAs of 148 SMs begin with: states in 32 bits 0.9 million, in 8 bits 4.8 million)
@pytest.mark.parametrize("tensors", [20, 130])
@pytest.mark.parametrize("kind,elements", [("32bit", 5 * 10 ** 6), ("nearest", 16 * 10 ** 6), ("random", 16 * 10 ** 6)])
def test_many_chunks(kind, elements, tensors):
    from paper_2303_11257_b200 import lib as L
    eight = kind != "32bit"
    cases = _cases(tensors, elements, eight, tensors)
    assert sum(c.p.size for c in cases) > (8 if eight else 2) * 10 ** 6
    plan = L.adamw_tensors([c.dev_p for c in cases], [c.dev_g for c in cases], [c.state[0] for c in cases], [c.state[1] for c in cases], [c.scales[0] for c in cases],
                           [c.scales[1] for c in cases], [c.copy for c in cases], 1.0, [c.decay for c in cases], 1.0, L.US_ROUND_RANDOM if kind == "random" else L.US_ROUND_NEAREST)
    step = L.new_adamw_step()
    for t in (1, 2):
        before = [(U.host_values(c.dev_p).ravel(),) + c.held() for c in cases]
        L.us_adamw(plan, step, 0.01)
        torch.cuda.synchronize()
        assert step.tolist() == [t, 0]
        for k, (c, b) in enumerate(zip(cases, before)):
            if kind == "random":
                if t == 2 or c.p.size < 10 ** 5:                   # (the oracle's codes of large tensors take long)
                    _check_codes(c, b, t, (k, c.shape, t))
                w = O.adamw_step(b[0], c.g.ravel(), b[1], b[2], t, 0.01, weight_decay=c.decay)
                assert np.allclose(U.host_values(c.dev_p).ravel(), w.p, rtol=1e-5, atol=1e-6)
            else:
                c.check(b, t, 0.01, what=(k, c.shape, t))
            if eight:
                _check_scales(c, b, (k, c.shape, t))


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("shape,kw", [((1, 77), {}), ((1, 300), {}), ((9, 130), dict(pads=(4, 4, 0))), ((9, 130), dict(shifts=(1, 0, 0, 0, 0))), ((5, 256), dict(shifts=(0, 0, 1, 2, 0))), ((40, 512), {})])
def test_scales_of_every_block(shape, kw, rounding):
    """Short last blocks, padded and unaligned tensors too."""
    from paper_2303_11257_b200 import lib as L
    c = Case(*shape, eight=True, grad="bf16", **kw)
    plan = L.adamw_tensors([c.dev_p], [c.dev_g], [c.state[0]], [c.state[1]], [c.scales[0]], [c.scales[1]], rounding=rounding)
    step = L.new_adamw_step()
    for t in (1, 2, 3):
        before = (U.host_values(c.dev_p).ravel(),) + c.held()
        L.us_adamw(plan, step, 0.01)
        _check_scales(c, before, (shape, t))
