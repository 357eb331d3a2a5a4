"""us_ffn_gated_fwd / us_ffn_gated_bwd against the oracle.

Tolerances.  A product sums K terms in float32 on the tensor core, each sum off by at most one step of 2^-23 of the magnitudes: with
S = scale * sum |x| |w| it is off by e = (K + 2) 2^-23 S.  The gate is evaluated with a relative error below 3e-6 (|z| 2^-23 |log2 e| + some
2^-22 for |z| <= 12, which no input here exceeds) or 1e-6 absolutely (tanh, gelu near their zero), both taken: f off by 3e-6 |f| + 1e-6.  A slope of f is at most 1.13.  So
A is off by alpha_g (1.13 s e_h |u| + |f| e_u + (3e-6 |f| + 1e-6) |u|) and a few 2^-24 |A|, which the 3e-6 covers; gradients likewise.  (relu's slope jumps at 0, in the
backward pass at the stored h, which both sides read.)  What is stored adds half a step of its format."""
import numpy as np
import pytest
import torch

from oracle import formats as F
from oracle import ops as O
from oracle import scales as S
from tests import util as U

pytestmark = pytest.mark.gpu
US_ERR_TIMEOUT = 6
# One shape per form of the launch on 148 SMs, ragged in every dimension: narrow tiles, wide ones of single CTAs, tiles of CTA pairs (one and
# several each, of short and of long contractions), both directions; single rows; a contraction longer than the ring of stages; the smallest matrices.
SHAPES = {"one": (1, 1, 1, 1), "token": (1, 520, 1104, 304), "few": (37, 144, 336, 208), "narrow": (300, 80, 1000, 144), "wide": (600, 272, 1500, 96), "wider": (600, 272, 2100, 96), "pair": (1300, 272, 1808, 400),
          "pairs": (2300, 96, 4870, 64), "deep": (1300, 1168, 1700, 64), "long": (130, 3000, 90, 2500), "tall": (5000, 33, 70, 65)}


def _lib():
    from paper_2303_11257_b200 import lib, synth
    return lib, synth


def _pitch(k):
    return (k + 15) // 16 * 16


def _close(got, ref, tol, fmt, what):
    g, top = U.host_values(got), F.FORMATS[fmt].max_finite
    if fmt in ("e4m3", "e5m2"):
        ref = np.clip(ref, -top, top)
    lim = tol + 0.5 * U.ulp_of(np.abs(ref) + tol, fmt) * (1 + 1e-6)
    bad = ~(np.abs(g - ref) <= lim)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.abs(g - ref)[bad].max()))


def _untouched(t, cols):
    raw = t.view(torch.uint8) if t.element_size() == 1 else t
    full = torch.as_strided(raw, (t.shape[0], t.stride(0)), (t.stride(0), 1))
    assert not full[:, cols:].any()


def _forward(shape, fn, fmt, kept, s_in=1.0, seed=0, fx=None, out=None, halves=True):
    L, synth = _lib()
    b, m, f, _ = shape
    fx, out = fx or fmt, out or fmt
    X, Wg, Wu = synth.normal(seed, 0, (b, m)), synth.normal(seed, 1, (m, f)), synth.normal(seed, 2, (m, f))
    Xt = U.to_device(X, fx, _pitch(m))
    W = U.empty(m, 2 * _pitch(f), fmt)
    Wt = (W[:, :f], W[:, _pitch(f):_pitch(f) + f]) if halves else (U.empty(m, f, fmt, _pitch(f)), U.empty(m, f, fmt, _pitch(f) + 32))
    for t, w in zip(Wt, (Wg, Wu)):
        t.copy_(U.to_device(w, fmt))
    alpha, a_out = m ** -0.5, 1.625
    A, ws = U.empty(b, f, out, _pitch(f) + 16), L.new_workspace()
    H, V = (U.empty(b, f, kept, _pitch(f) + 16) for _ in range(2)) if kept else (None, None)
    L.us_ffn_gated_fwd(fn, Xt, *Wt, alpha, A, ws, H=H, U=V, act_in_scale=s_in, act_out_scale=a_out)
    assert L.us_workspace_status(ws) == 0
    x, g, u = U.values_of(X, fx), U.values_of(Wg, fmt), U.values_of(Wu, fmt)
    ref, h, uu = O.gated_fwd(fn, x, g, u, alpha, s_in, a_out)
    eh, eu = ((m + 2) * 2.0 ** -23 * alpha * (np.abs(x) @ np.abs(w)) for w in (g, u))
    fv = np.abs(O.activation_fwd(fn, h, s_in, 1.0))
    assert np.abs(s_in * h).max() < 12
    _close(A, ref, a_out * (1.13 * s_in * eh * np.abs(uu) + fv * eu + (3e-6 * fv + 1e-6) * np.abs(uu)), out, "A")
    _untouched(A, f)
    if kept:
        _close(H, h, eh, kept, "H")
        _close(V, uu, eu, kept, "U")
        _untouched(H, f)
        _untouched(V, f)


def _backward(shape, fn, act, grad, kept, s_in=1.0, seed=0, out=None, in_place=False, big=1.0):
    L, synth = _lib()
    b, _, f, n = shape
    out = out or grad
    G, W2, H, V = synth.normal(seed, 3, (b, n)), synth.normal(seed, 4, (f, n)), synth.normal(seed, 5, (b, f)) * np.float32(big), synth.normal(seed, 6, (b, f))
    Gt, Wt = U.to_device(G, grad, _pitch(n)), U.to_device(W2, act, _pitch(n) + 16)
    Ht, Vt = U.to_device(H, kept, _pitch(f) + 16), U.to_device(V, kept, _pitch(f) + 16)
    dH, dU = (Ht.view(U.TORCH_OF[out]), Vt.view(U.TORCH_OF[out])) if in_place else (U.empty(b, f, out, _pitch(f)), U.empty(b, f, out, _pitch(f) + 16))
    ws, beta_x, bh, bu = L.new_workspace(), n ** -0.5, 1.5, 1.25
    L.us_ffn_gated_bwd(fn, Gt, Wt, beta_x, Ht, Vt, dH, dU, ws, act_in_scale=s_in, beta_h=bh, beta_u=bu)
    assert L.us_workspace_status(ws) == 0
    g, w, h, u = U.values_of(G, grad), U.values_of(W2, act), U.values_of(H, kept), U.values_of(V, kept)
    rh, ru = O.gated_bwd(fn, g, w, beta_x, h, u, s_in, bh, bu)
    d = O.linear_bwd_x(g, w, beta_x)
    e = (n + 2) * 2.0 ** -23 * beta_x * (np.abs(g) @ np.abs(w).T)
    fv, df = np.abs(O.activation_fwd(fn, h, s_in, 1.0)), np.abs(O.activation_bwd(fn, h, np.ones_like(h), s_in, 1.0)) / s_in
    _close(dU, ru, bu * (fv * e + (3e-6 * fv + 1e-6) * np.abs(d)), out, "dU")
    _close(dH, rh, bh * s_in * np.abs(u) * (df * e + (3e-6 * df + 2e-6) * np.abs(d)), out, "dH")
    if not in_place:
        _untouched(dU, f)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("fmt,kept", [("bf16", "bf16"), ("fp16", "fp16"), ("e4m3", "e4m3"), ("e4m3", None)])
def test_forward(shape, fmt, kept):
    _forward(SHAPES[shape], "silu", fmt, kept)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("act,grad,kept", [("bf16", "bf16", "bf16"), ("fp16", "fp16", "e4m3"), ("e4m3", "e5m2", "e4m3"), ("e4m3", "e5m2", "bf16")])
def test_backward(shape, act, grad, kept):
    _backward(SHAPES[shape], "silu", act, grad, kept)


@pytest.mark.parametrize("fn", ["gelu", "relu", "tanh", "sigmoid", "silu"])
@pytest.mark.parametrize("s_in", [1.0, 0.625])
@pytest.mark.parametrize("shape", ["few", "pair"])
def test_every_gate(fn, s_in, shape):
    for fmt, grad in (("fp16", "fp16"), ("e4m3", "e5m2")):
        _forward(SHAPES[shape], fn, fmt, "fp16", s_in, seed=1)
        _backward(SHAPES[shape], fn, fmt, grad, "fp16", s_in, seed=1)


@pytest.mark.parametrize("shape", ["few", "wide", "pair"])
def test_every_mix_of_formats(shape):
    for fmt, fx, out, kept in (("e5m2", "e4m3", "e5m2", "fp16"), ("e4m3", "e5m2", "e4m3", "bf16"), ("bf16", None, None, "e4m3"), ("fp16", None, None, "bf16"), ("bf16", None, None, None)):
        _forward(SHAPES[shape], "silu", fmt, kept, seed=2, fx=fx, out=out, halves=False)
    for act, grad, out, kept in (("e5m2", "e4m3", "e4m3", "fp16"), ("e4m3", "e4m3", "e5m2", "e4m3"), ("bf16", "bf16", None, "e4m3"), ("bf16", "bf16", None, "fp16"), ("fp16", "fp16", None, "bf16")):
        _backward(SHAPES[shape], "silu", act, grad, kept, seed=2, out=out)


@pytest.mark.parametrize("shape", ["token", "narrow", "wide", "pairs"])
def test_gradients_in_the_place_of_the_copies(shape):
    _backward(SHAPES[shape], "silu", "bf16", "bf16", "bf16", in_place=True)
    _backward(SHAPES[shape], "silu", "e4m3", "e5m2", "e4m3", in_place=True)


def test_copies_saturate_and_far_values_keep_their_limits():
    """f of far arguments: 0 or z, slopes 0 or 1; E4M3 copies of more than 448 are 448."""
    L, _ = _lib()
    b, f, ws = 200, 96, L.new_workspace()
    X = torch.ones(b, 16, device="cuda").bfloat16()
    Wg, Wu = torch.full((16, f), 60.0, device="cuda").bfloat16(), torch.ones(16, f, device="cuda").bfloat16()
    Wg[:, 1::2] = -60.0
    A, H, V = (torch.empty(b, f, device="cuda", dtype=d) for d in (torch.bfloat16, torch.float8_e4m3fn, torch.float8_e4m3fn))
    L.us_ffn_gated_fwd("silu", X, Wg, Wu, 1.0, A, ws, H=H, U=V)                    # h = +-960, u = 16
    assert (A[:, ::2] == 15360).all() and (A[:, 1::2] == 0).all() and (H.float()[:, ::2] == 448).all() and (H.float()[:, 1::2] == -448).all() and (V.float() == 16).all()
    dH, dU = torch.empty_like(A), torch.empty_like(A)
    L.us_ffn_gated_bwd("silu", X, torch.ones(f, 16, device="cuda").bfloat16(), 1.0, H, V, dH, dU, ws)      # dA = 16
    assert (dH[:, ::2] == 256).all() and (dH[:, 1::2] == 0).all() and (dU[:, ::2] == 7168).all() and (dU[:, 1::2] == 0).all()
    assert L.us_workspace_status(ws) == 0


@pytest.mark.parametrize("shape", ["token", "few", "wide", "pair"])
def test_values_that_are_not_finite_stay_in_their_row_or_column(shape):
    L, synth = _lib()
    b, m, f, n = SHAPES[shape]
    bf = lambda i, r, c: U.to_device(synth.normal(9, i, (r, c)), "bf16", _pitch(c))
    X, Wg, Wu, G, W2, H, V = bf(0, b, m), bf(1, m, f), bf(2, m, f), bf(3, b, n), bf(4, f, n), bf(5, b, f), bf(6, b, f)
    ws = L.new_workspace()
    out = lambda: U.empty(b, f, "bf16", _pitch(f))

    def both():
        A, h, u, dH, dU = (out() for _ in range(5))
        L.us_ffn_gated_fwd("silu", X, Wg, Wu, m ** -0.5, A, ws, H=h, U=u)
        L.us_ffn_gated_bwd("silu", G, W2, n ** -0.5, H, V, dH, dU, ws)
        assert L.us_workspace_status(ws) == 0
        return A, h, u, dH, dU
    clean = both()
    X[b - 1, 0], Wu[0, 7], G[b - 1, 1], V[0, 3] = float("nan"), float("inf"), float("nan"), float("nan")
    A, h, u, dH, dU = both()
    ok = torch.ones(b, f, dtype=torch.bool, device="cuda")
    ok[b - 1] = False
    assert torch.isnan(h[b - 1]).all() and torch.isnan(A[b - 1]).all() and torch.isnan(dU[b - 1]).all()
    assert torch.equal(h[ok], clean[1][ok]) and torch.equal(dU[ok], clean[4][ok])
    ok[:, 7] = False
    assert torch.equal(u[ok], clean[2][ok]) and torch.equal(A[ok], clean[0][ok]) and (b == 1 or torch.isinf(u[0, 7]))
    ok[:, 7] = True
    ok[b - 1] = False
    ok[0, 3] = False
    assert torch.equal(dH[ok], clean[3][ok]) and torch.isnan(dH[0, 3])


@pytest.mark.parametrize("shape", ["token", "wide", "pairs"])
def test_captured_replayed_and_on_another_stream(shape):
    """Two graphs and an eager pass that share a workspace, each on new values in the same tensors: the same bits."""
    L, synth = _lib()
    b, m, f, n = SHAPES[shape]
    e4 = lambda i, r, c: U.to_device(synth.normal(11, i, (r, c)), "e4m3", _pitch(c))
    X, Wg, Wu, G, W2 = e4(0, b, m), e4(1, m, f), e4(2, m, f), e4(3, b, n), e4(4, f, n)
    ws, sets = L.new_workspace(), [[U.empty(b, f, k, _pitch(f)) for k in ("e4m3", "e4m3", "e4m3", "e5m2", "e5m2")] for _ in range(3)]

    def step(A, H, V, dH, dU):
        L.us_ffn_gated_fwd("silu", X, Wg, Wu, m ** -0.5, A, ws, H=H, U=V)
        L.us_ffn_gated_bwd("silu", G, W2, n ** -0.5, H, V, dH, dU, ws)
    step(*sets[0])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, s in zip(graphs, sets):
        with torch.cuda.graph(g):
            step(*s)
    X.copy_(e4(7, b, m))
    G.copy_(e4(8, b, n))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(streams[0]):
        graphs[0].replay()
    with torch.cuda.stream(streams[1]):
        graphs[1].replay()
    torch.cuda.synchronize()
    step(*sets[2])
    torch.cuda.synchronize()
    assert L.us_workspace_status(ws) == 0
    for i in range(5):
        assert torch.equal(sets[0][i].contiguous().view(torch.uint8), sets[1][i].contiguous().view(torch.uint8))
        assert torch.equal(sets[0][i].contiguous().view(torch.uint8), sets[2][i].contiguous().view(torch.uint8))


@pytest.mark.parametrize("shape", ["few", "narrow", "wide", "wider", "pair", "pairs"])   # (but for "wider" forward and backward take the same kind of tile)
def test_starved_launches_time_out_and_the_next_call_is_correct(shape):
    L, synth = _lib()
    b, m, f, n = SHAPES[shape]
    e4 = lambda i, r, c: U.to_device(synth.normal(13, i, (r, c)), "e4m3", _pitch(c))
    X, Wg, Wu, G, W2, H, V = e4(0, b, m), e4(1, m, f), e4(2, m, f), e4(3, b, n), e4(4, f, n), e4(5, b, f), e4(6, b, f)
    ws, outs = L.new_workspace(), [U.empty(b, f, "e4m3", _pitch(f)) for _ in range(5)]

    def run():
        L.us_ffn_gated_fwd("silu", X, Wg, Wu, 0.1, outs[0], ws, H=outs[1], U=outs[2])
        L.us_ffn_gated_bwd("silu", G, W2, 0.1, H, V, outs[3], outs[4], ws)
        assert L.us_workspace_status(ws) == 0
        return [o.contiguous().view(torch.uint8).clone() for o in outs]
    want = run()
    for cta, tiles in ((-1, 0), (-1, 1), (0, 0), (1, 0), (1, 1)):
        if cta >= 0 and (shape == "wider" or (cta == 1) != shape.startswith("pair")):          # of a CTA pair the odd one, whose copies the even one waits for
            continue
        for starve in (lambda: L.us_test_ffn_gated_fwd_starved(X, Wg, Wu, outs[1], outs[2], outs[0], ws, 2000, cta, tiles),
                       lambda: L.us_test_ffn_gated_bwd_starved(G, W2, H, V, outs[3], outs[4], ws, 2000, cta, tiles)):
            starve()
            if tiles == 0 or shape == "pairs":
                assert L.us_workspace_status(ws) == US_ERR_TIMEOUT, (cta, tiles)
            torch.cuda.synchronize()
            ws.zero_()
            assert all(torch.equal(a, b) for a, b in zip(run(), want))


def test_the_even_cta_of_a_pair_does_not_starve_alone():
    """Nobody would wait for the copies of the odd one: the hook refuses it where tiles are a pair's."""
    L, _ = _lib()
    b, m, f, n = SHAPES["pair"]
    X, Wg, Wu, A, ws = U.empty(b, 272, "e4m3"), U.empty(m, f, "e4m3"), U.empty(m, f, "e4m3"), U.empty(b, f, "e4m3"), L.new_workspace()
    with pytest.raises(L.UnitScaleError) as e:
        L.us_test_ffn_gated_fwd_starved(X, Wg, Wu, None, None, A, ws, 2000, 0, 0)
    assert e.value.status == 1
    with pytest.raises(L.UnitScaleError) as e:
        L.us_test_ffn_gated_bwd_starved(U.empty(b, n, "e4m3"), U.empty(f, n, "e4m3"), A, A, U.empty(b, f, "e4m3"), U.empty(b, f, "e4m3"), ws, 2000, 0, 0)
    assert e.value.status == 1 and L.us_workspace_status(ws) == 0


def test_silu_as_an_elementwise_op():
    """us_activation_fwd / bwd: float32 results within 4e-7 of the definition, relative to 1 + |z|."""
    L, _ = _lib()
    H = torch.linspace(-20, 20, 4001, device="cuda").view(1, -1)
    dA, A, dH = torch.full_like(H, 0.5), torch.empty_like(H), torch.empty_like(H)
    L.us_activation_fwd("silu", H, 0.75, 1.5, A)
    L.us_activation_bwd("silu", H, dA, 0.75, 1.25, dH)
    h = H.double().cpu().numpy()
    assert np.all(np.abs(A.double().cpu().numpy() - O.activation_fwd("silu", h, 0.75, 1.5)) <= 1.5 * 4e-7 * (1 + np.abs(h)))
    assert np.all(np.abs(dH.double().cpu().numpy() - O.activation_bwd("silu", h, 0.5, 0.75, 1.25)) <= 4e-7 * (1 + np.abs(h)))
    assert all(abs(a - b) < 1e-6 for a, b in zip(L.us_scales_activation("silu"), S.silu_scales()))


def _gate_and_slope(fn, z):
    """f and f' for sigmoid and tanh, in closed forms without cancellation."""
    if fn == "sigmoid":
        e = np.exp(-np.abs(z))
        return np.where(z >= 0, 1.0, e) / (1 + e), e / (1 + e) ** 2
    return np.tanh(z), np.cosh(z) ** -2.0


def _gradients_of_both_signs(b, f, act, grad, kept, s_in, fn):
    """(z, dH, dU) for arguments from 2^-12 to 15 in the left half of the columns and their negatives in the right one; u = dA = 1 exactly."""
    L, _ = _lib()
    v = np.float32(2.0 ** np.linspace(-12, np.log2(15), b * (f // 2))).reshape(b, -1)
    h = U.values_of(np.concatenate([v, -v], 1), kept)
    Ht, Vt = U.to_device(np.float32(h), kept, _pitch(f)), U.to_device(np.ones((b, f), np.float32), kept, _pitch(f))
    one = lambda r, fmt: U.to_device(np.float32(np.eye(1, 16)).repeat(r, 0), fmt)                 # rows (1, 0, 0 ..)
    dH, dU, ws = U.empty(b, f, grad, _pitch(f)), U.empty(b, f, grad, _pitch(f)), L.new_workspace()
    L.us_ffn_gated_bwd(fn, one(b, grad), one(f, act), 1.0, Ht, Vt, dH, dU, ws, act_in_scale=s_in)
    assert L.us_workspace_status(ws) == 0
    return s_in * h, dH, dU


SIGNED = [(b, f, *types) for b, f in ((37, 336), (1300, 1808)) for types in (("bf16", "bf16", "fp16"), ("fp16", "fp16", "bf16"), ("e4m3", "e5m2", "e4m3"), ("e4m3", "e5m2", "fp16"))]


@pytest.mark.parametrize("fn", ["sigmoid", "tanh"])
@pytest.mark.parametrize("s_in", [1.0, 0.625])
@pytest.mark.parametrize("case", SIGNED)
def test_slopes_near_zero_and_far_from_it(case, s_in, fn):
    """Errors relative to the slope s (1 - s) itself (tanh: 4 s (1 - s) of 2 z).  In units of 2^-24: e = 2^(-z log2 e) (tanh: of 2 z) is off by 5 |z| from the rounded product and
    4 from ex2; s = 1 / (1 + e) by 3 and e / (1 + e) of that; 1 - s = e s by what is left of it, 1 / (1 + e), 3 and 1; so with its products the slope by
    5 |z| + 17; 6 |z| + 32 is taken."""
    z, dH, _ = _gradients_of_both_signs(*case, s_in, fn)
    slope = s_in * _gate_and_slope(fn, z)[1]
    _close(dH, slope, (6 * np.abs(z) + 32) * 2.0 ** -24 * slope, case[3], "dH")


@pytest.mark.parametrize("fn", ["sigmoid", "tanh"])
@pytest.mark.parametrize("s_in", [1.0, 0.625])
@pytest.mark.parametrize("case", SIGNED)
def test_values_near_zero_and_far_from_it(case, s_in, fn):
    """The gate's values, in dU and in A, with errors relative to the value itself.  In units of 2^-24: s = sigmoid(z) is off by 5 |z| + 7 (as above); tanh from 1/8 on, as 2 s - 1
    with s of 2 z, by 2 s (3 + (1 - s) (5 |z| + 4)) and 1, 9 at 1/8, where that is 8 times as much of the value, and 5 where |z| is large; below 1/8, as a polynomial, by the term left out, 4, and
    five roundings; products 5.  6 |z| + 96 is taken."""
    b, f, act, grad, kept = case
    L, _ = _lib()
    z, _, dU = _gradients_of_both_signs(*case, s_in, fn)
    value = _gate_and_slope(fn, z)[0]
    _close(dU, value, (6 * np.abs(z) + 96) * 2.0 ** -24 * np.abs(value), grad, "dU")
    h = np.float32(2.0 ** np.linspace(-12, np.log2(15), f // 2))
    h = U.values_of(np.concatenate([h, -h])[None], act)
    rows = lambda r: U.to_device(np.float32(np.concatenate([r, np.zeros((15, f))])), act, _pitch(f))
    X, A, ws = U.to_device(np.float32(np.eye(1, 16)).repeat(b, 0), act), U.empty(b, f, act, _pitch(f)), L.new_workspace()
    L.us_ffn_gated_fwd(fn, X, rows(h), rows(np.ones((1, f))), 1.0, A, ws, act_in_scale=s_in)
    assert L.us_workspace_status(ws) == 0
    z = s_in * h
    value = _gate_and_slope(fn, z)[0].repeat(b, 0)
    _close(A, value, (6 * np.abs(z) + 96) * 2.0 ** -24 * np.abs(value), act, "A")


@pytest.mark.parametrize("fn", ["gelu", "relu", "tanh", "sigmoid", "silu"])
@pytest.mark.parametrize("shape", ["token", "pair"])
def test_every_gate_keeps_a_nan(fn, shape):
    L, synth = _lib()
    b, m, f, n = SHAPES[shape]
    bf = lambda i, r, c: U.to_device(synth.normal(17, i, (r, c)), "bf16", _pitch(c))
    X, Wg, Wu, G, W2, H, V = bf(0, b, m), bf(1, m, f), bf(2, m, f), bf(3, b, n), bf(4, f, n), bf(5, b, f), bf(6, b, f)
    Wg[0, 5] = H[0, 3] = float("nan")
    A, dH, dU = (U.empty(b, f, "bf16", _pitch(f)) for _ in range(3))
    ws = L.new_workspace()
    L.us_ffn_gated_fwd(fn, X, Wg, Wu, m ** -0.5, A, ws)
    L.us_ffn_gated_bwd(fn, G, W2, n ** -0.5, H, V, dH, dU, ws)
    assert L.us_workspace_status(ws) == 0
    nan = torch.isnan(A)
    assert nan[:, 5].all() and int(nan.sum()) == b
    assert all(torch.isnan(t[0, 3]) and int(torch.isnan(t).sum()) == 1 for t in (dH, dU))


@pytest.mark.parametrize("fn", ["sigmoid", "tanh"])
@pytest.mark.parametrize("act,grad", [("bf16", "bf16"), ("e4m3", "e5m2")])
def test_limits_of_sigmoid_and_tanh(fn, act, grad):
    """Arguments of +-100, +-1e30 and infinity: the limits, with slopes of nothing, and no NaN."""
    L, _ = _lib()
    b, f, ws = 40, 96, L.new_workspace()
    h = torch.tensor([100.0, 1e30, float("inf")] * 16, device="cuda")
    H = torch.cat([h, -h]).expand(b, f).contiguous().bfloat16()
    one = lambda r, fmt: U.to_device(np.float32(np.eye(1, 16)).repeat(r, 0), fmt)
    dH, dU = U.empty(b, f, grad), U.empty(b, f, grad)
    L.us_ffn_gated_bwd(fn, one(b, grad), one(f, act), 1.0, H, torch.ones_like(H), dH, dU, ws)
    low = 0.0 if fn == "sigmoid" else -1.0
    assert (dH.float() == 0).all() and (dU.float()[:, :48] == 1).all() and (dU.float()[:, 48:] == low).all()
    if act == "bf16":                                             # (8-bit operands have no infinities)
        X, Wg, Wu, A = one(b, act), U.empty(16, f, act), U.empty(16, f, act), U.empty(b, f, act)
        Wg[0], Wu[0] = H[0].clamp(-1e38, 1e38), 1.0
        L.us_ffn_gated_fwd(fn, X, Wg, Wu, 10.0, A, ws)             # (infinities by the scale: an infinite weight times a zero of X is NaN)
        assert (A.float()[:, :48] == 10).all() and (A.float()[:, 48:] == 10 * low).all()          # u = 10, too
    assert L.us_workspace_status(ws) == 0
