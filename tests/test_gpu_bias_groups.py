"""Biases in the launches that hold several products: us_ffn_hidden_bias and us_linear_group_bias against the calls of one product each, bit for bit where these sum
in the same order, and against sums in 64 bits where they do not."""
import numpy as np
import pytest
import torch

from oracle import ops as O
from tests import util as U
from tests.test_gpu_ffn_hidden import FORMS

pytestmark = pytest.mark.gpu
PAD = lambda c: (c + 15) // 16 * 16
BIAS = {"f32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _bits(t):
    return t.contiguous().view(torch.uint8)


# beside the forms of a tile: one row, columns that end inside a warp's part, several tiles per unit (a tile's biases follow the last one's)
HIDDEN = {**FORMS, "row": (1, 16, 33, 16), "ragged": (129, 80, 135, 208), "tiles": (2304, 256, 4871, 256), "singles": (1152, 64, 2063, 80)}


@pytest.mark.parametrize("form", HIDDEN)
@pytest.mark.parametrize("act,grad,h_fmt,bias,keep", [("e4m3", "e5m2", "bf16", "f32", False), ("e5m2", "e4m3", "fp16", "bf16", True), ("bf16", "bf16", "bf16", "fp16", True),
                                                      ("fp16", "fp16", "fp16", "f32", False)])
def test_hidden_layer_equals_the_separate_calls(form, act, grad, h_fmt, bias, keep):
    from paper_2303_11257_b200 import lib as L, synth
    b, m, f, n = HIDDEN[form]
    ws = L.new_workspace()
    dev = lambda i, s, fmt: U.to_device(synth.normal(9, i, s), fmt, PAD(s[1]))
    X, W1, G, W2 = dev(0, (b, m), act), dev(1, (m, f), act), dev(2, (b, n), grad), dev(3, (f, n), act)
    B = torch.from_numpy(synth.normal(9, 4, (1, f + 1)) * 2.0).cuda().to(BIAS[bias])[0, 1:]          # not on a boundary of 16 bytes
    out = lambda fmt: U.empty(b, f, fmt, PAD(f))
    A, dH, H, A1, dH1, H1 = out(act), out(grad), out(h_fmt), out(act), out(grad), out(h_fmt)
    L.us_ffn_hidden_bias(X, W1, m ** -0.5, B, G, W2, n ** -0.5, 0.75, 1.7, 1.48, A, dH, ws, H=H if keep else None, h_dtype=H.dtype)
    L.us_linear_fwd_bias(X, W1, m ** -0.5, B, A1, ws, L.epilogue(act=L.US_ACT_GELU, act_in_scale=0.75, act_out_scale=1.7, aux=H1))
    L.us_linear_bwd_x(G, W2, n ** -0.5, dH1, ws, L.epilogue(act=L.US_ACT_GELU_GRAD, act_in_scale=0.75, act_out_scale=1.48, aux=H1))
    assert L.us_workspace_status(ws) == 0
    for a, r in ((A, A1), (dH, dH1)) + (((H, H1),) if keep else ()):
        assert np.array_equal(U.codes_of(a), U.codes_of(r))
    if form in ("two", "ragged"):
        ref = O.linear_bias_fwd(U.host_values(X), U.host_values(W1), m ** -0.5, U.host_values(B).reshape(-1))
        U.assert_close_stored(H1, ref, h_fmt, 2e-3 * max(1.0, np.abs(ref).max() / 4), "pre-activation")


# pair tiles, 128 x 128 tiles, two CTAs a tile; the last two: shared contractions in a second launch, with the forward product among the sharing ones and not
GROUPS = {"pair": (1200, 400, 1200), "single": (700, 272, 1031), "split": (200, 144, 400), "row": (1, 16, 48), "forward shares": (48, 1024, 7000), "forward does not": (9000, 128, 304)}


@pytest.mark.parametrize("form", GROUPS)
@pytest.mark.parametrize("act,grad,out,bias", [("e4m3", "e5m2", "bf16", "f32"), ("bf16", "bf16", "f32", "fp16"), ("fp16", "fp16", "fp16", "bf16")])
def test_group(form, act, grad, out, bias):
    from paper_2303_11257_b200 import lib as L, synth
    T, d, f = GROUPS[form]
    ws = L.new_workspace()
    dev = lambda i, s, fmt: U.to_device(synth.normal(10, i, s) * (np.arange(s[1]) >= (16 if i == 2 else 0)), fmt, PAD(s[1]))
    # (columns of zeros in the gradient: products of zero, which a negative scale makes -0)
    Aq, W2, Gq, Xq, dH, S = dev(0, (T, f), act), dev(1, (f, d), act), dev(2, (T, d), grad), dev(3, (T, d), act), dev(4, (T, f), grad), dev(5, (T, d), out)
    B = torch.from_numpy(synth.normal(10, 6, (1, d + 1)) * 2.0).cuda().to(BIAS[bias])[0, 1:]
    ep = L.epilogue(skip=S, skip_coef=0.8, out_coef=0.6)

    def outs():
        return U.empty(T, d, out, PAD(d)), U.empty(f, d, "f32", PAD(d)), U.empty(d, f, "f32", PAD(f))

    def calls(R, dW2, dW1):
        return [L.linear_call(L.US_OP_BWD_W, Aq, Gq, -0.1, dW2), L.linear_call(L.US_OP_BWD_W, Xq, dH, 0.1, dW1), L.linear_call(L.US_OP_FWD, Aq, W2, f ** -0.5, R, ep)]
    got, plain, again = outs(), outs(), outs()
    L.us_linear_group_bias(calls(*got), [None, None, B], ws)
    L.us_linear_group_any(calls(*plain), ws)
    assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(got[1:], plain[1:]))
    assert bool((got[1] == 0).any()) and bool(torch.signbit(got[1][got[1] == 0]).all())
    assert L.us_linear_group_launches(calls(*got)) == (2 if form.startswith("forward") else 1)
    for _ in range(2):
        L.us_linear_group_bias(calls(*again), [None, None, B], ws)
        assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(got, again))
    assert L.us_workspace_status(ws) == 0
    if form == "forward shares":
        # sums in eight chains or more of at most f products: f / 16 roundings of 2^-24 of the sum of magnitudes, and the output's own
        a, w = U.host_values(Aq), U.host_values(W2)
        branch = f ** -0.5 * (a @ w) + U.host_values(B).reshape(1, -1)
        ref = 0.8 * U.host_values(S) + 0.6 * branch
        eps = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "f32": 2.0 ** -22}[out]
        tol = 0.6 * (f / 16) * 2.0 ** -24 * f ** -0.5 * (np.abs(a) @ np.abs(w)) + eps * np.abs(ref) + 1e-6
        assert (np.abs(U.host_values(got[0]) - ref) <= tol).all()
    else:
        single = outs()[0]
        L.us_linear_fwd_bias(Aq, W2, f ** -0.5, B, single, ws, ep)
        assert torch.equal(_bits(got[0]), _bits(single))


def test_a_refused_group_adds_its_biases_in_single_launches():
    """More tiles than the work list holds: the prepared group goes out as single launches."""
    from paper_2303_11257_b200 import lib as L, synth
    n, k, ws = 46 * 256, 16, L.new_workspace()
    X, W, B = U.to_device(synth.normal(60, 0, (n, k)), "e4m3"), U.to_device(synth.normal(60, 1, (k, n)), "e4m3"), torch.from_numpy(synth.normal(60, 2, (1, n))).cuda()[0]
    Y, Y1 = U.empty(n, n, "bf16"), U.empty(n, n, "bf16")
    call = L.Plan((), ()).group([(L.US_OP_FWD, X, W, 0.25, Y, Y, (0.0, 1.0))], ws, biases={0: B})
    call(L.current_stream())
    assert call.refused
    L.us_linear_fwd_bias(X, W, 0.25, B, Y1, ws)
    assert L.us_workspace_status(ws) == 0 and torch.equal(Y.view(torch.int16), Y1.view(torch.int16))
