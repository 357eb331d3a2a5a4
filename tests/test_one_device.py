"""Linear ops with biases, gradients of biases, gradient norms and optimiser steps take CUDA tensors of one device, the current one: every argument is looked at, on the host."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2303_11257_b200 import lib as L

F32, BF = L.US_F32, L.US_BF16
without_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls with fake addresses")


def M(addr, dt, r, c):
    return L.us_mat(addr, dt, r, c, c)


def _calls():
    """name -> arguments that the library takes (fake addresses), and those of them that may be tensors."""
    X, W, Y, b = M(0x10000, BF, 8, 64), M(0x20000, BF, 64, 64), M(0x30000, BF, 8, 64), M(0x40000, F32, 1, 64)
    ws = (0x50000, 4096)
    one = (L.us_mat * 1)(M(0x10000, F32, 8, 64))
    call = (L.us_linear_call * 1)()
    call[0].a, call[0].b, call[0].out, call[0].scale = X, W, Y, 1.0
    return {"us_linear_fwd_bias": ([X, W, 1.0, b, None, Y, None, *ws, 0], (0, 1, 3, 5, 7)),
            "us_ffn_hidden_bias": ([X, W, 1.0, b, X, W, 1.0, 1.0, 1.0, 1.0, BF, None, Y, Y, *ws, 0], (0, 1, 3, 4, 5, 11, 12, 13, 14)),
            "us_linear_group_bias": ([1, call, (L.us_mat * 1)(b), *ws, 0], (3,)),
            "us_bias_grad": ([1, one, None, (L.us_mat * 1)(b), 0], ([1], [3])),
            "us_grad_norm": ([1, one, 1.0, 0x60000, 0x50000, 1 << 16, 0], ([1], 3, 4)),
            "us_adamw": ([1, (L.us_adamw_tensor * 1)(), 1e-3, 0.9, 0.999, 1e-8, None, None, 0x70000, 0], (6, 7, 8))}


HOST = [torch.zeros(8, 64), torch.zeros(64)]


@without_gpu
@pytest.mark.parametrize("name", sorted(_calls()))
def test_tensors_in_host_memory_are_refused_wherever_they_stand(name):
    args, places = _calls()[name]
    assert L._entry(name)(*args) in (1, 5)                        # (1: the empty tensor of us_adamw; 5: no device)
    for at in places:
        for t in HOST:
            other = list(args)
            other[at[0] if isinstance(at, list) else at] = [t] if isinstance(at, list) else t
            with pytest.raises(ValueError):
                L._entry(name)(*other)


def test_tensors_of_two_devices_are_not_laid_out_together(monkeypatch):
    device = {}

    def fill(address, stride, tensors):
        there = {device[id(t)] for t in tensors if t is not None}
        return there.pop() if there else -1
    monkeypatch.setattr(L._binding, "fill", fill)
    p, g, m, v = (torch.zeros(4) for _ in range(4))
    for t in (p, g, m, v):
        device[id(t)] = 0
    assert L.adamw_tensors([p], [g], [m], [v])._device == 0 and L.mats([g])._device == 0 and L.mats([])._device == -1
    for t in (p, g, m, v):
        device[id(t)] = 1
        with pytest.raises(ValueError, match="one device"):
            L.adamw_tensors([p], [g], [m], [v])
        device[id(t)] = 0


class OnDevice:
    """What the wrappers ask of a tensor."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, dtype, n=2):
        self.dtype, self.n = dtype, n

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0


def test_what_was_laid_out_on_another_device_is_refused(monkeypatch):
    monkeypatch.setattr(L, "_current_device", lambda: 0)
    for arr, call in (((L.us_adamw_tensor * 1)(), lambda a: L.us_adamw(a, OnDevice(torch.int64), 1e-3)),
                      ((L.us_mat * 1)(), lambda a: L.us_grad_norm(a, 1.0, OnDevice(torch.float32), None))):
        arr._device = 1
        with pytest.raises(ValueError, match="laid out on device 1"):
            call(arr)


@pytest.mark.parametrize("which", range(6))
def test_tensors_of_epilogues_and_groups_are_looked_at(monkeypatch, which):
    """Those that their descriptions were made of: kept pre-activation and skip tensor, operands and results."""
    monkeypatch.setattr(L, "_current_device", lambda: 0)
    monkeypatch.setattr(L, "describe", lambda t: (0x10000, BF, 8, 64, 64))
    monkeypatch.setattr(L, "_entry", lambda name: lambda *a: 0)
    monkeypatch.setattr(L, "_stream", lambda stream: 0)
    t = [OnDevice(BF) for _ in range(6)]
    X, W, Y, H, S, ws = t

    def calls():
        ep = L.epilogue(act=L.US_ACT_GELU, aux=t[3], skip=t[4])
        L.us_linear_fwd_bias(X, W, 1.0, None, t[2], ws, ep)
        L.us_linear_group_bias([L.linear_call(L.US_OP_FWD, t[0], t[1], 1.0, t[2], L.epilogue(skip=t[4]))], [None], t[5])
    calls()
    t[which] = torch.zeros(8, 64)
    with pytest.raises(ValueError, match="current CUDA device"):
        calls()


@pytest.mark.gpu
def test_host_memory_beside_device_memory():
    on = lambda *s: torch.ones(*s, device="cuda")
    x, w, y, b, ws = on(8, 64).bfloat16(), on(64, 64).bfloat16(), on(8, 64).bfloat16(), on(64), L.new_workspace()
    for ep in (L.epilogue(act=L.US_ACT_GELU, aux=y.cpu()), L.epilogue(skip=y.cpu(), skip_coef=0.5, out_coef=0.5)):
        with pytest.raises(ValueError):
            L.us_linear_fwd_bias(x, w, 1.0, b, y, ws, ep)
    for args in ((x.cpu(), w, 1.0, b, y, ws), (x, w.cpu(), 1.0, b, y, ws), (x, w, 1.0, b.cpu(), y, ws), (x, w, 1.0, b, y, ws.cpu())):
        with pytest.raises(ValueError):
            L.us_linear_fwd_bias(*args)
    with pytest.raises(ValueError):
        L.us_bias_grad([x.cpu()], None, [b])
    with pytest.raises(ValueError):
        L.us_grad_norm([x.cpu()], 1.0, on(2), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        L.us_grad_norm([x], 1.0, on(2), torch.zeros(1 << 16, dtype=torch.uint8))
    with pytest.raises(ValueError):
        L.adamw_tensors([on(4)], [torch.ones(4)], [on(4)], [on(4)])
    L.us_linear_fwd_bias(x, w, 1.0, b, y, ws)                      # (and all of it on the device)
    assert torch.equal(y.float(), torch.full_like(y, 65.0).float())


WITHOUT_ASSERTIONS = """
import torch
from paper_2303_11257_b200 import lib as L
from tests.test_one_device import OnDevice
L._current_device = lambda: 0
arr, mats, step, out = (L.us_adamw_tensor * 1)(), (L.us_mat * 1)(), OnDevice(torch.int64), OnDevice(torch.float32)
bad = [lambda: L.us_adamw(arr, OnDevice(torch.int32), 1e-3), lambda: L.us_adamw(arr, OnDevice(torch.int64, 1), 1e-3), lambda: L.us_grad_norm(mats, 1.0, OnDevice(torch.float32, 1), None),
       lambda: L.us_grad_norm(mats, 1.0, OnDevice(torch.float64), None), lambda: L.us_adamw(arr, step, 1e-3, lr_factor=OnDevice(torch.float32, 0)),
       lambda: L.us_adamw(arr, step, 1e-3, grad_factor=OnDevice(torch.float64)), lambda: L.us_adamw(arr, step, 1e-3, grad_factor=OnDevice(torch.float32, 0))]
for i, call in enumerate(bad):
    try:
        call()
    except AssertionError:
        continue
    except Exception as e:
        print(i, type(e).__name__, e)
    raise SystemExit(f"call {i} was not refused")
"""


@pytest.mark.parametrize("options", [[], ["-O"]])
def test_arguments_are_looked_at_without_assertions_too(options):
    """Records of other types and sizes, and factors without an element, which would be taken for none."""
    r = subprocess.run([sys.executable, *options, "-c", WITHOUT_ASSERTIONS], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stdout + r.stderr
