"""What us_qk_norm_fwd / bwd and us_rotary_table refuse, on the host, before anything is launched (1 invalid argument, 2 unsupported,
3 alignment, 4 workspace, 5 no device: everything else was in order); fake device addresses."""
import ctypes as C

import pytest
import torch

from paper_2303_11257_b200 import _binding
from paper_2303_11257_b200 import lib as L

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls with fake addresses")
BF, F32, E4 = L.US_BF16, L.US_F32, L.US_E4M3


def M(addr, dt, r, c, ld=None):
    return L.us_mat(addr, dt, r, c, c if ld is None else ld)


def arr(*ms):
    return (L.us_mat * len(ms))(*ms)


TABLE = M(0x90000, F32, 32, 64)


def fwd(X=M(0x10000, BF, 8, 256), w=M(0x20000, F32, 1, 64), Y=M(0x30000, BF, 8, 256), width=64, eps=1e-6, table=TABLE, pos=None, start=0, period=0, nb=0, count=1):
    return _binding.calls["us_qk_norm_fwd"](count, arr(X), None if w is None else arr(w), arr(Y), width, eps, table, pos, start, period, nb, 0)


def test_forward():
    assert fwd() == 5 and fwd(w=None) == 5 and fwd(table=None) == 5 and fwd(w=M(None, 0, 0, 0)) == 5 and fwd(table=M(None, 0, 0, 0)) == 5
    assert fwd(pos=0x40000, table=M(0x90000, F32, 1, 64)) == 5
    for bad in (dict(count=0), dict(width=0), dict(width=63), dict(eps=-1.0), dict(eps=float("nan")), dict(start=-1), dict(period=-1), dict(nb=2), dict(Y=M(0x30000, BF, 8, 128)),
                dict(Y=M(0x30000, BF, 7, 256)), dict(Y=M(0x30000, 9, 8, 256)), dict(X=M(0x10000, BF, 8, 256, 255)), dict(X=M(None, BF, 8, 256)), dict(w=M(0x20000, F32, 1, 65)),
                dict(w=M(0x20000, F32, 2, 64)), dict(table=M(0x90000, F32, 32, 63)), dict(table=M(0x90000, F32, 32, 66)), dict(table=M(0x90000, F32, 7, 64)),
                dict(table=M(0x90000, F32, 0, 64), pos=0x40000), dict(start=25), dict(period=4, start=29)):
        assert fwd(**bad) == 1, bad
    assert fwd(period=4, start=28) == 5 and fwd(start=24) == 5
    wide = dict(X=M(0x10000, BF, 8, 2048), w=None, Y=M(0x30000, BF, 8, 2048), width=2048)
    for bad in (dict(X=M(0x10000, E4, 8, 256)), dict(w=M(0x20000, E4, 1, 64)), dict(table=M(0x90000, BF, 32, 64)), wide):
        assert fwd(**bad) == 2, bad
    for bad in (dict(X=M(0x10001, BF, 8, 256)), dict(Y=M(0x30002, F32, 8, 256)), dict(w=M(0x20002, F32, 1, 64)), dict(table=M(0x90002, F32, 32, 64)), dict(pos=0x40002)):
        assert fwd(**bad) == 3, bad
    five = arr(*[M(0x10000, BF, 8, 256)] * 5)
    assert _binding.calls["us_qk_norm_fwd"](5, five, None, five, 64, 0.0, None, None, 0, 0, 0, 0) == 1


def bwd(X=M(0x10000, BF, 8, 256), w=M(0x20000, F32, 1, 64), G=M(0x50000, BF, 8, 256), dX=M(0x30000, L.US_E5M2, 8, 256), dw=M(0x60000, F32, 1, 64), ws=0x70000, size=1 << 20):
    raw = L.raw().us_qk_norm_bwd
    one = lambda m: None if m is None else arr(m)
    return raw(1, one(X), one(w), one(G), one(dX), one(dw), None, 64, 0.0, 1.0, C.byref(TABLE), None, 0, 0, 0, ws, size, None)


def test_backward():
    need = L.us_qk_norm_bwd_workspace_bytes(64)
    assert need > 0 and L.us_qk_norm_bwd_workspace_bytes(1025) == 0 and L.us_qk_norm_bwd_workspace_bytes(0) == 0
    assert bwd() == 5 and bwd(dw=None, ws=None, size=0) == 5 and bwd(w=None, dw=None) == 5 and bwd(size=need) == 5
    assert bwd(G=None) == 1 and bwd(G=M(0x50000, BF, 8, 128)) == 1 and bwd(w=None) == 1 and bwd(dw=M(0x60000, F32, 1, 63)) == 1
    assert bwd(G=M(0x50000, E4, 8, 256)) == 2 and bwd(dw=M(0x60000, E4, 1, 64)) == 2
    assert bwd(G=M(0x50001, BF, 8, 256)) == 3 and bwd(ws=0x70008) == 3
    assert bwd(ws=None) == 4 and bwd(size=need - 1) == 4


def test_table():
    t = _binding.calls["us_rotary_table"]
    assert t(TABLE, 10000.0, 1.0, 0, 0) == 5 and t(M(0x90000, F32, 0, 64), 10000.0, 1.0, 0, 0) == 0 and t(M(0x90000, F32, 4, 0), 10000.0, 1.0, 0, 0) == 0
    for bad in ((None, 10.0, 1.0, 0), (TABLE, 0.0, 1.0, 0), (TABLE, 10.0, -1.0, 0), (TABLE, 10.0, float("nan"), 0), (TABLE, 10.0, 1.0, -1), (M(0x90000, F32, 4, 3), 10.0, 1.0, 0)):
        assert t(*bad, 0) == 1, bad
    assert t(M(0x90000, BF, 4, 4), 10.0, 1.0, 0, 0) == 2 and t(M(0x90002, F32, 4, 4), 10.0, 1.0, 0, 0) == 3


def test_lists_of_tensors_are_described_by_the_binding():
    x, w = torch.zeros(4, 128, dtype=torch.bfloat16), torch.ones(64)
    call = _binding.calls["us_qk_norm_fwd"]
    assert call(2, [x, x], [w, None], (x, x), 64, 0.0, None, None, 0, 0, 0, 0) == 5
    assert call(1, [x], [torch.ones(63)], [x], 64, 0.0, None, None, 0, 0, 0, 0) == 1
    for bad, error in (([x], ValueError), ([x, 5], TypeError), ([x, torch.zeros(16, 8).t()], ValueError), ([x, torch.zeros(2, 2, dtype=torch.int64)], KeyError), ([x] * 33, ValueError),
                       ([x, torch.ones(128)[::2]], ValueError)):
        with pytest.raises(error):
            call(2, bad, None, [x, x], 64, 0.0, None, None, 0, 0, 0, 0)
    with pytest.raises(TypeError):                                # a prepared call outlives the lists
        _binding.prepare("us_qk_norm_fwd", (1, [x], None, [x], 64, 0.0, None, None, 0, 0, 0))
    for numbers, error in (([1.0], ValueError), ([1.0, "a"], TypeError), ([1.0] * 17, ValueError)):
        with pytest.raises(error):
            _binding.calls["us_qk_norm_bwd"](2, [x, x], None, [x, x], [x, x], None, numbers, 64, 0.0, 1.0, None, None, 0, 0, 0, None, 0, 0)
    with pytest.raises(ValueError):
        L.us_qk_norm_fwd([x, x], [w], [x, x], 64, 0.0, stream=0)
    with pytest.raises(AssertionError):
        L.us_qk_norm_fwd([x], None, [x], 64, 0.0, positions=torch.zeros(4), stream=0)


def test_starts_near_the_end_of_64_bits():
    """start + rows is not formed where it would pass 2^63."""
    last = 2 ** 63 - 1
    for start in (last, last - 3, last - 7, 2 ** 62, 2 ** 32, 2 ** 32 + 3):
        assert fwd(start=start) == 1 and fwd(start=start, period=4) == 1 and fwd(start=start, period=1) == 1, start
    assert fwd(period=last) == 5 and fwd(period=last, start=24) == 5 and fwd(period=last, start=25) == 1
    # where the positions are on the device, or nothing is turned, start is not read
    assert fwd(start=last, pos=0x40000) == 5 and fwd(start=last, table=None) == 5


def test_positions_in_host_memory():
    """The kernels would read them through an address that is none on the device."""
    x, at = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(AssertionError):
        L.us_qk_norm_fwd([x], None, [x], 64, 0.0, positions=at, stream=0)
    with pytest.raises(AssertionError):
        L.us_qk_norm_bwd([x], None, [x], [x], None, 64, 0.0, None, positions=at, stream=0)
