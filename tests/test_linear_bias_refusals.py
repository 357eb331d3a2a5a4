"""What us_linear_fwd_bias refuses on the host (1 invalid argument, 2 unsupported, 3 alignment, 4 workspace, 5 no device: all else in order)."""
import ctypes as C

import pytest
import torch

from paper_2303_11257_b200 import lib as L

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls with fake addresses")
BF, F16, F32, E4, E5 = L.US_BF16, L.US_F16, L.US_F32, L.US_E4M3, L.US_E5M2


def M(addr, dt, r, c, ld=None):
    return L.us_mat(addr, dt, r, c, c if ld is None else ld)


def call(X=M(0x10000, BF, 8, 64), W=M(0x20000, BF, 64, 48), bias=M(0x30000, F32, 1, 48), ep=None, Y=M(0x40000, BF, 8, 48), Yq=None, ws=0x70000, size=256):
    ref = lambda m: None if m is None else C.byref(m)
    return L.raw().us_linear_fwd_bias(ref(X), ref(W), 0.5, ref(bias), ref(ep), ref(Y), ref(Yq), ws, size, None)


def ep(act=0, aux=None, skip=None):
    e = L.us_epilogue()
    e.act, e.act_in_scale, e.act_out_scale, e.out_coef, e.skip_coef = act, 1.0, 1.0, 1.0, 1.0
    if aux is not None:
        e.aux = aux
    if skip is not None:
        e.skip = skip
    return e


SKIP, Q = M(0x50000, F32, 8, 48), M(0x60000, E4, 8, 48)


def test_what_is_taken():
    for dt in (F32, BF, F16):
        assert call(bias=M(0x30000, dt, 1, 48)) == 5 and call(bias=M(0x30000, dt, 1, 48, 50)) == 5
    for act in (L.US_ACT_GELU, L.US_ACT_RELU, L.US_ACT_TANH, L.US_ACT_SIGMOID):
        assert call(ep=ep(act)) == 5 and call(ep=ep(act, aux=M(0x50000, BF, 8, 48))) == 5 and call(ep=ep(act, skip=SKIP)) == 5
    assert call(ep=ep(skip=SKIP)) == 5 and call(ep=ep(skip=SKIP), Yq=Q) == 5


def test_what_is_refused():
    for bad in (None, M(None, F32, 1, 48), M(0x30000, F32, 1, 47), M(0x30000, F32, 2, 48), M(0x30000, F32, 48, 1), M(0x30000, 9, 1, 48), M(0x30000, F32, 1, 48, 47)):
        assert call(bias=bad) == 1
    assert call(X=M(0x10000, BF, 8, 63)) == 1 and call(Y=M(0x40000, BF, 7, 48)) == 1
    for bad in (E4, E5):
        assert call(bias=M(0x30000, bad, 1, 48)) == 2
    for act in (L.US_ACT_GELU_GRAD, L.US_ACT_RELU_GRAD, L.US_ACT_TANH_GRAD, L.US_ACT_SIGMOID_GRAD):
        assert call(ep=ep(act, aux=M(0x50000, BF, 8, 48))) == 2
    assert call(Yq=Q) == 2 and call(ep=ep(L.US_ACT_GELU, skip=SKIP), Yq=Q) == 2 and call(ep=ep(skip=SKIP), Yq=M(0x60000, BF, 8, 48)) == 2
    assert call(X=M(0x10000, F16, 8, 64)) == 2
    assert call(bias=M(0x30002, F32, 1, 48)) == 3 and call(bias=M(0x30001, BF, 1, 48)) == 3 and call(bias=M(0x30004, F32, 1, 48)) == 5 and call(bias=M(0x30002, F16, 1, 48)) == 5
    assert call(ws=None) == 4 and call(size=255) == 4 and call(ws=0x70008) == 3


def hidden(bias=M(0x30000, F32, 1, 48), X=M(0x10000, E4, 200, 64), H=None, h_dtype=BF, ws=0x70000):
    ref = lambda m: None if m is None else C.byref(m)
    T = X.rows
    fmt = X.dtype
    return L.raw().us_ffn_hidden_bias(ref(X), ref(M(0x20000, fmt, 64, 48)), 0.5, ref(bias), ref(M(0x80000, fmt, T, 32)), ref(M(0x90000, fmt, 48, 32)), 0.5, 1.0, 1.0, 1.0,
                                      h_dtype, ref(H), ref(M(0xa0000, fmt, T, 48)), ref(M(0xb0000, fmt, T, 48)), ws, 256, None)


def test_hidden_layer():
    for dt in (F32, BF, F16):
        for fmt in (E4, BF, F16):
            assert hidden(bias=M(0x30000, dt, 1, 48, 50), X=M(0x10000, fmt, 200, 64)) == 5
    for bad in (None, M(None, F32, 1, 48), M(0x30000, F32, 1, 47), M(0x30000, F32, 2, 48), M(0x30000, F32, 48, 1), M(0x30000, 9, 1, 48), M(0x30000, F32, 1, 48, 47)):
        assert hidden(bias=bad) == 1
    assert hidden(h_dtype=F32) == 1 and hidden(H=M(0xc0000, F16, 200, 48)) == 1
    for bad in (E4, E5):
        assert hidden(bias=M(0x30000, bad, 1, 48)) == 2
    assert hidden(X=M(0x10000, F32, 200, 64)) == 2
    assert hidden(bias=M(0x30002, F32, 1, 48)) == 3 and hidden(bias=M(0x30001, BF, 1, 48)) == 3 and hidden(bias=M(0x30002, BF, 1, 48)) == 5
    assert hidden(ws=None) == 4 and hidden(ws=0x70008) == 3


def group(biases, op=L.US_OP_FWD, count=2, act=0):
    calls = (L.us_linear_call * 2)()
    for c in calls:
        c.op, c.a, c.b, c.scale, c.out, c.ep = L.US_OP_FWD, M(0x10000, BF, 48, 48), M(0x20000, BF, 48, 48), 0.5, M(0x40000, BF, 48, 48), ep(act)
    calls[1].op = op
    return L.raw().us_linear_group_bias(count, calls, None if biases is None else (L.us_mat * 2)(*biases), 0x70000, 256, None)


def test_group():
    none, good = L.us_mat(), M(0x30000, F32, 1, 48)
    for biases in ([none, none], [none, good], [good, good], [M(0x30002, BF, 1, 48), none]):
        assert group(biases) == 5
    assert group([good, none], op=L.US_OP_BWD_X) == 5 and group([good, none], op=L.US_OP_BWD_W) == 5
    for op in (L.US_OP_BWD_X, L.US_OP_BWD_W):
        assert group([none, good], op=op) == 1
    for bad in (M(0x30000, F32, 1, 47), M(0x30000, F32, 48, 1), M(0x30000, 9, 1, 48)):
        assert group([none, bad]) == 1
    assert group(None) == 1 and group([none, good], count=0) == 1 and group([none, good], count=5) == 2
    assert group([none, M(0x30000, E4, 1, 48)]) == 2 and group([none, good], act=L.US_ACT_GELU) == 2
    assert group([none, M(0x30002, F32, 1, 48)]) == 3
