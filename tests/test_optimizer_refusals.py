"""What us_adamw, us_grad_norm and us_bias_grad refuse, on the host, before anything is launched (1 invalid argument, 2 unsupported, 3 alignment,
4 workspace, 5 no device: everything else was in order); fake device addresses."""
import ctypes as C
import math

import pytest
import torch

from paper_2303_11257_b200 import lib as L

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls with fake addresses")
BF, F16, F32, E4, E5 = L.US_BF16, L.US_F16, L.US_F32, L.US_E4M3, L.US_E5M2


def M(addr, dt, r, c, ld=None):
    return L.us_mat(addr, dt, r, c, c if ld is None else ld)


def tensor(param=M(0x10000, F32, 8, 100), grad=M(0x20000, BF, 8, 100), m=M(0x30000, F32, 1, 800), v=M(0x40000, F32, 800, 1), m_scale=None, v_scale=None,
           copy=M(0x50000, E4, 8, 100, 128), numbers=(1.0, 1.0, 0.0)):
    t = L.us_adamw_tensor()
    for name, x in dict(param=param, grad=grad, m=m, v=v, m_scale=m_scale, v_scale=v_scale, copy=copy).items():
        if x is not None:
            setattr(t, name, x)
    t.copy_scale, t.lr_factor, t.weight_decay = numbers
    return t


def adamw(*ts, count=None, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, lr_factor=None, grad_factor=None, step=0x90000):
    arr = (L.us_adamw_tensor * max(1, len(ts)))(*ts)
    return L.raw().us_adamw(len(ts) if count is None else count, arr, lr, b1, b2, eps, lr_factor, grad_factor, step, None)


EIGHT = dict(m=M(0x30000, E4, 8, 100), v=M(0x40000, E4, 8, 100), m_scale=M(0x60000, F32, 1, 4), v_scale=M(0x70000, F32, 4, 1))


def test_adamw():
    assert adamw(tensor()) == 5 and adamw(tensor(copy=None)) == 5 and adamw(tensor(**EIGHT)) == 5 and adamw(tensor(), tensor(**EIGHT)) == 5
    assert adamw(tensor(), lr_factor=0xa0000, grad_factor=0xa0004) == 5 and adamw(tensor(), lr=0.0, b1=0.0, b2=0.0) == 5
    assert adamw(tensor(param=M(0x10004, F32, 8, 100, 101), grad=M(0x20002, F16, 8, 100, 103), m=M(0x30004, F32, 8, 100), copy=M(0x50001, E5, 8, 100, 111))) == 5
    assert adamw(tensor(param=M(0x10000, F32, 8, 100, 99))) == 1
    for bad in (dict(count=0), dict(step=None), dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(b1=1.0), dict(b1=-0.1), dict(b2=math.nan), dict(b2=1.0),
                dict(eps=0.0), dict(eps=1e-60), dict(eps=-1.0), dict(eps=math.nan), dict(eps=1e60)):
        assert adamw(tensor(), **bad) == 1, bad
    for bad in (dict(grad=M(0x20000, BF, 100, 8)), dict(m=M(0x30000, F32, 1, 801)), dict(v=M(0x30000, F32, 1, 799)), dict(copy=M(0x50000, E4, 8, 99)), dict(param=M(None, F32, 8, 100)),
                dict(grad=M(None, BF, 8, 100)), dict(copy=M(0x50000, 7, 8, 100)), dict(copy=M(0x50000, E4, 8, 100, 99)), dict(numbers=(math.nan, 1.0, 0.0)),
                dict(numbers=(1.0, math.inf, 0.0)), dict(numbers=(1.0, 1.0, math.nan)), {**EIGHT, "m_scale": M(0x60000, F32, 1, 3)}, {**EIGHT, "v_scale": None}):
        assert adamw(tensor(), tensor(**bad)) == 1, bad
    for bad in (dict(param=M(0x10000, BF, 8, 100)), dict(grad=M(0x20000, E5, 8, 100)), dict(m=M(0x30000, BF, 8, 100), v=M(0x30000, BF, 8, 100)), dict(m=M(0x30000, E4, 8, 100)),
                dict(m=M(0x30000, F32, 8, 100, 104)), {**EIGHT, "v": M(0x40000, E4, 8, 100, 112)}, {**EIGHT, "m_scale": M(0x60000, BF, 1, 4)},
                {**EIGHT, "v_scale": M(0x70000, F32, 4, 1, 2)}):
        assert adamw(tensor(**bad)) == 2, bad
    for bad in (dict(param=M(0x10002, F32, 8, 100)), dict(grad=M(0x20001, BF, 8, 100)), dict(v=M(0x40001, F32, 8, 100)), dict(copy=M(0x50001, BF, 8, 100)),
                {**EIGHT, "m_scale": M(0x60002, F32, 1, 4)}):
        assert adamw(tensor(**bad)) == 3, bad
    assert adamw(tensor(), step=0x90004) == 3 and adamw(tensor(), lr_factor=0xa0002) == 3 and adamw(tensor(), grad_factor=0xa0001) == 3
    none = M(None, F32, 0, 100)
    assert adamw(tensor(param=none, grad=M(None, BF, 0, 100), m=none, v=none, copy=None)) == 5      # a step without elements is counted


def norm(*ms, count=None, most=1.0, out=0x80000, ws=0x90000, size=1 << 20):
    return L.raw().us_grad_norm(len(ms) if count is None else count, (L.us_mat * max(1, len(ms)))(*ms), most, out, ws, size, None)


def test_grad_norm():
    g, need = M(0x10000, F32, 8, 100, 101), L.us_grad_norm_workspace_bytes()
    assert norm(g) == 5 and norm(g, M(0x20002, BF, 1, 7), M(None, F16, 0, 5)) == 5 and norm(g, most=math.inf) == 5 and norm(g, size=need) == 5
    for bad in (dict(count=0), dict(most=0.0), dict(most=-1.0), dict(most=math.nan), dict(out=None)):
        assert norm(g, **bad) == 1, bad
    assert norm(M(None, F32, 8, 100)) == 1 and norm(M(0x10000, F32, 8, 100, 99)) == 1 and norm(M(0x10000, 6, 8, 100)) == 1
    assert norm(M(0x10000, E5, 8, 100)) == 2 and norm(g, M(0x10000, E4, 8, 100)) == 2
    assert norm(M(0x10002, F32, 8, 100)) == 3 and norm(g, out=0x80002) == 3 and norm(g, ws=0x90008) == 3
    assert norm(g, ws=None) == 4 and norm(g, size=need - 1) == 4


def bias(*pairs, count=None, beta=True):
    n = len(pairs)
    mats = lambda k: (L.us_mat * max(1, n))(*[p[k] for p in pairs])
    return L.raw().us_bias_grad(n if count is None else count, mats(0), (C.c_float * max(1, n))() if beta else None, mats(1), None)


def test_bias_grad():
    G, db = M(0x10000, E5, 8, 100, 112), M(0x20000, F32, 1, 100)
    assert bias((G, db)) == 5 and bias((G, db), beta=False) == 5 and bias(*[(G, db)] * 8) == 5 and bias((M(0x10001, E4, 8, 100, 101), M(0x20002, BF, 1, 100))) == 5
    assert bias((M(None, BF, 0, 100), db)) == 5 and bias((M(None, BF, 5, 0), M(None, F32, 1, 0))) == 0     # (nothing to be written)
    assert bias(*[(G, db)] * 9) == 1 and bias((G, db), count=0) == 1
    for bad in ((M(None, E5, 8, 100), db), (M(0x10000, E5, 8, 100, 99), db), (M(0x10000, 5, 8, 100), db), (G, M(0x20000, F32, 1, 99)), (G, M(0x20000, F32, 2, 100)),
                (G, M(None, F32, 1, 100)), (M(0x10000, E5, -1, 100), db)):
        assert bias((G, db), bad) == 1, bad
    assert bias((G, M(0x20000, E4, 1, 100))) == 2
    assert bias((M(0x10001, BF, 8, 100), db)) == 3 and bias((G, M(0x20002, F32, 1, 100))) == 3


def test_python_side():
    t = torch.zeros(4)
    with pytest.raises(ValueError):
        L.adamw_tensors([t], [t], [t], [t, t])
    with pytest.raises(ValueError):
        L.adamw_tensors([t], [t], [t], [t])                       # host memory
    with pytest.raises(ValueError):
        L.us_bias_grad([t], [1.0], [])
    with pytest.raises(ValueError):
        L.us_bias_grad([t.view(1, 4)], [1.0], [t])
    with pytest.raises(ValueError):
        L.us_linear_fwd_bias(t.view(1, 4), t.view(4, 1), 1.0, t[:1], t[:1].view(1, 1), t)
    with pytest.raises(AssertionError):
        L.us_adamw(None, torch.zeros(2, dtype=torch.int64), 1e-3)
    with pytest.raises(AssertionError):
        L.us_grad_norm([], 1.0, torch.zeros(2), None)
