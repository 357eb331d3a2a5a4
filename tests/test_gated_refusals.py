"""What us_ffn_gated_fwd / bwd refuse, on the host, before anything is launched (1 invalid argument, 2 unsupported, 3 alignment,
4 workspace, 5 no device: everything else was in order); fake device addresses."""
import ctypes as C

import pytest
import torch

from paper_2303_11257_b200 import lib as L

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls with fake addresses")
BF, F16, F32, E4, E5 = L.US_BF16, L.US_F16, L.US_F32, L.US_E4M3, L.US_E5M2


def M(dt, r, c, ld=None, addr=0x10000):
    return L.us_mat(addr, dt, r, c, c if ld is None else ld)


def ref(m):
    return None if m is None else C.byref(m)


def fwd(fn=4, dt=E4, X=None, Wg=None, Wu=None, H=None, U=None, A=None, ws=0x20000, size=4096):
    X, Wg, Wu, A = X or M(dt, 300, 64), Wg or M(dt, 64, 208), Wu or M(dt, 64, 208), A or M(dt, 300, 208)
    return L.raw().us_ffn_gated_fwd(fn, ref(X), ref(Wg), ref(Wu), 1.0, 1.0, 1.0, ref(H), ref(U), ref(A), ws, size, None)


def bwd(fn=4, dt=E4, G=None, W2=None, H=None, U=None, dH=None, dU=None, ws=0x20000, size=4096):
    G, W2 = G or M(dt, 300, 64), W2 or M(dt, 208, 64)
    H, U, dH, dU = H or M(BF, 300, 208), U or M(BF, 300, 208), dH or M(dt, 300, 208), dU or M(dt, 300, 208)
    return L.raw().us_ffn_gated_bwd(fn, ref(G), ref(W2), 1.0, 1.0, 1.0, 1.0, ref(H), ref(U), ref(dH), ref(dU), ws, size, None)


K = M(BF, 300, 208)


def test_what_is_in_order():
    for dt in (E4, BF, F16):
        for kept in (None, BF, F16, E4):
            k = None if kept is None else M(kept, 300, 208)
            assert fwd(dt=dt, H=k, U=k) == 5
            assert kept is None or bwd(dt=dt, H=k, U=k) == 5
    assert fwd(X=M(E5, 300, 64)) == 5 and fwd(Wg=M(E5, 64, 208), Wu=M(E5, 64, 208)) == 5 and fwd(A=M(E5, 300, 208)) == 5 and fwd(H=M(0, 0, 0, addr=None), U=None) == 5
    assert bwd(G=M(E5, 300, 64), dH=M(E5, 300, 208), dU=M(E5, 300, 208)) == 5


def test_forward():
    for bad in (dict(fn=5), dict(fn=-1), dict(X=M(E4, 300, 80)), dict(Wu=M(E4, 64, 224)), dict(Wu=M(E4, 80, 208)), dict(Wu=M(E5, 64, 208)), dict(A=M(E4, 300, 224)), dict(A=M(E4, 299, 208)),
                dict(H=K), dict(U=K), dict(H=K, U=M(F16, 300, 208)), dict(H=K, U=M(BF, 300, 200)), dict(H=M(BF, 299, 208), U=M(BF, 299, 208)), dict(X=M(E4, 0, 64)),
                dict(X=M(E4, 300, 64, 48)), dict(X=M(E4, 300, 64, addr=None)), dict(X=M(7, 300, 64))):
        assert fwd(**bad) == 1, bad
    for bad in (dict(dt=F32), dict(A=M(BF, 300, 208)), dict(X=M(BF, 300, 64)), dict(dt=BF, A=M(F16, 300, 208)), dict(dt=BF, A=M(E4, 300, 208)), dict(dt=BF, X=M(F16, 300, 64)),
                dict(H=M(F32, 300, 208), U=M(F32, 300, 208)), dict(H=M(E5, 300, 208), U=M(E5, 300, 208))):
        assert fwd(**bad) == 2, bad
    huge = (1 << 31) - 1
    assert fwd(X=M(E4, huge, 64), A=M(E4, huge, 208)) == 2 and fwd(X=M(E4, 300, huge, 1 << 31), Wg=M(E4, huge, 208), Wu=M(E4, huge, 208)) == 2
    for bad in (dict(X=M(E4, 300, 64, 72)), dict(Wu=M(E4, 64, 208, addr=0x10008)), dict(A=M(E4, 300, 208, 216)), dict(H=K, U=M(BF, 300, 208, 212)), dict(ws=0x20008)):
        assert fwd(**bad) == 3, bad
    assert fwd(ws=None) == 4 and fwd(size=L.us_workspace_bytes() - 1) == 4


def test_backward():
    for bad in (dict(fn=5), dict(W2=M(E4, 208, 80)), dict(W2=M(E4, 224, 64)), dict(H=M(BF, 300, 200)), dict(U=M(F16, 300, 208)), dict(dU=M(E5, 300, 208)), dict(dH=M(E4, 301, 208)),
                dict(H=M(BF, 300, 208, addr=None))):
        assert bwd(**bad) == 1, bad
    assert L.raw().us_ffn_gated_bwd(4, None, None, 1.0, 1.0, 1.0, 1.0, None, None, None, None, None, 0, None) == 1
    for bad in (dict(dt=F32), dict(G=M(BF, 300, 64)), dict(dH=M(BF, 300, 208), dU=M(BF, 300, 208)), dict(H=M(F32, 300, 208), U=M(F32, 300, 208)),
                dict(H=M(E5, 300, 208), U=M(E5, 300, 208))):
        assert bwd(**bad) == 2, bad
    for bad in (dict(G=M(E4, 300, 64, 72)), dict(H=M(BF, 300, 208, 212), U=K), dict(dU=M(E4, 300, 208, addr=0x10004)), dict(ws=0x20001)):
        assert bwd(**bad) == 3, bad
    assert bwd(ws=None) == 4 and bwd(size=1) == 4


def test_starved_forms_check_their_limits():
    m = [ref(M(E4, 300, 64)), ref(M(E4, 64, 208)), ref(M(E4, 64, 208)), None, None, ref(M(E4, 300, 208))]
    b = [ref(M(E4, 300, 64)), ref(M(E4, 208, 64)), ref(K), ref(K), ref(M(E4, 300, 208)), ref(M(E4, 300, 208))]
    for name, args in (("us_test_ffn_gated_fwd_starved", m), ("us_test_ffn_gated_bwd_starved", b)):
        f = getattr(L.raw(), name)
        for limit, cta, tiles in ((0, -1, 0), (1 << 17, -1, 0), (100, -2, 0), (100, 2, 0), (100, 0, -1), (100, 0, 1025)):
            assert f(*args, 0x20000, 4096, limit, cta, tiles, None) == 1
        assert f(*args, 0x20000, 4096, 100, 0, 0, None) == 5
