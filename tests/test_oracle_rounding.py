"""The oracle's random rounding of states in 8 bits: the numbers, the codes, and what states become over many steps beside states that are not rounded."""
import numpy as np
import pytest

from oracle import formats as F
from oracle import ops as O


def test_fractions_are_even_and_independent():
    """Means, variances and correlations of 400 steps x 5000 elements: 2 million uniform numbers, whose mean is off by 1 / sqrt(12 n) = 2e-4 and whose correlations by n^-1/2 = 7e-4, of
    one element by 400^-1/2 = 0.05; five of these are allowed."""
    a = [O.rounding_bits(t, 5000) for t in range(1, 401)]
    for x in (np.array([m for m, _ in a]), np.array([r for _, r in a])):
        n = x.size
        assert x.min() >= 0 and x.max() < 1
        assert abs(x.mean() - 0.5) < 5 / np.sqrt(12 * n) and abs(x.var() - 1 / 12) < 1e-3
        assert np.abs(x.mean(0) - 0.5).max() < 5.5 / np.sqrt(12 * 400) and np.abs(x.mean(1) - 0.5).max() < 5 / np.sqrt(12 * 5000)
        y = (x - 0.5) * np.sqrt(12)
        for lag in (1, 2, 4, 128, 256):
            assert abs((y[:, lag:] * y[:, :-lag]).mean()) < 5 / np.sqrt(n)          # of neighbours
        for lag in (1, 2, 7):
            assert abs((y[lag:] * y[:-lag]).mean()) < 5 / np.sqrt(n)                # of steps
    m, r = (np.array(x) for x in zip(*a))
    assert abs(((m - 0.5) * (r - 0.5)).mean() * 12) < 5 / np.sqrt(m.size)
    assert not np.array_equal(O.rounding_bits(1, 9)[1], O.rounding_bits(2 ** 32 + 1, 9)[1])


def test_codes_are_around_their_values_and_keep_the_mean():
    rng = np.random.default_rng(0)
    x = np.concatenate([[448.0], rng.standard_normal(255) * 100, [448.0, 2.0 ** -6, 2.0 ** -9, -2.0 ** -10, 3.3 * 2.0 ** -9, 0.0, 1.0, -17.5, 440.0]]).clip(-448, 448)
    n, total = x.size, np.zeros(x.size)
    apart = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    for t in range(1, 2001):
        c, _ = O.block_codes(x, fractions=O.rounding_bits(t, n)[1])
        assert np.array_equal(F.quantise(c, F.FORMATS["e4m3"]), c) and (np.abs(c - x) < apart).all()
        total += c
    assert (np.abs(total / 2000 - x) <= 5 * apart * 0.5 / np.sqrt(2000) + 1e-12).all()        # (the variance of one is at most a quarter)
    c, _ = O.block_codes(np.array([1.0, 1e-9, 0.0]), positive=True, fractions=np.zeros(3))
    assert c[1] == 2.0 ** -9 and c[2] == 0.0


@pytest.mark.parametrize("fall", [0.1, 0.0])
def test_states_follow_their_averages_over_many_steps(fall):
    """Gradients of log-normal size; after 500 of 3500 steps those of every second element fall, to a tenth or to none.  With random rounding sqrt(v) keeps the mean that it has without
    rounding, and the mean step its size; to the nearest code sqrt(v) stays far above and the steps far below.

    A step changes sqrt(v) by up to 0.05 % of itself, so one of about 180 goes to another code, 9 % away: the square of the spread grows by 0.0005 x 0.09 = 4.5e-5 a step.  Where gradients
    keep their size it is forgotten at the rate 0.002 and stays at 0.0225: spread 0.15, and the mean square that rounding adds to v (4.5e-5 / 0.001 = 4.5 %) makes the mean sqrt(v) 1.1 % larger;
    1 / sqrt(v) is 1 + 0.15^2 times as large.  Means of 256 are off by 0.15 / 16: four of those and the bias, 0.05 and 0.06, taken as 0.06 and 0.07.  Where gradients have fallen nothing is forgotten for the
    3000 steps: 0.135, spread 0.37, four times 0.37 / 16 = 0.09 of the mean, taken as 0.1; of 1 / sqrt(v), 1 + 0.135 and as much, 0.23, taken as 0.25 (no gradients: no steps)."""
    n, falls, steps, lr = 512, 500, 3500, 1e-3
    found = {}
    for kind in ("none", "random", "nearest"):
        rng = np.random.default_rng(7)
        sigma = np.exp(rng.standard_normal(n))
        m, v, size = np.zeros(n), np.zeros(n), []
        for t in range(1, steps + 1):
            g = sigma * rng.standard_normal(n)
            if t > falls:
                g[::2] *= fall
            s = O.adamw_step(np.zeros(n), g, m, v, t, lr)
            m, v = s.m, s.v
            if kind != "none":
                a, b = O.rounding_bits(t, n) if kind == "random" else (None, None)
                (cm, sm), (cv, sv) = O.block_codes(m, fractions=a), O.block_codes(np.sqrt(v), positive=True, fractions=b)
                m, v = np.repeat(sm, 256) * cm, (np.repeat(sv, 256) * cv) ** 2
            if t > steps - 200:
                size.append(np.abs(s.update))
        found[kind] = np.sqrt(v), np.mean(size, 0)
    root, size = found["none"]
    for part, tol_root, tol_step in ((slice(0, None, 2), 0.1, 0.25), (slice(1, None, 2), 0.06, 0.07)):
        assert abs((found["random"][0][part] / root[part]).mean() - 1) < tol_root
        assert abs(found["random"][1][part].mean() - size[part].mean()) <= tol_step * size[part].mean() + 1e-9 * lr
    assert (found["nearest"][0][::2] / root[::2]).mean() > 2
    assert fall == 0 or found["nearest"][1][::2].mean() < 0.6 * size[::2].mean()
