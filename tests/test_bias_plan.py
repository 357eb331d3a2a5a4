"""What an FFN block with biases issues, without a GPU: the calls and their order, copies of a block, arguments that have to fit."""
import copy

import pytest
import torch

from paper_2303_11257_b200 import ffn, optim
from paper_2303_11257_b200 import lib as L
from tests.test_gated_plan import _Recorder


def _ffn(**kw):
    return ffn.UnitScaledBiasFFN(64, 32, 48, device="cpu", **kw), [torch.zeros(s) for s in ((64, 32), (32, 48), (48, 32), (64, 32))]


@pytest.mark.parametrize("operand", ["fp8", "bf16"])
def test_calls_of_a_step(monkeypatch, operand):
    block, x = _ffn(operand=operand)
    rec = _Recorder()
    monkeypatch.setattr(L, "_lib", rec)
    gemms = ["ffn_hidden_bias", "bias_grad", "linear_group_bias"]
    apart = ["linear_fwd_bias", "linear_fwd_bias", "linear_bwd_x", "bias_grad", "linear_group_any"]
    block.step(*x, stream=0)
    assert rec.names() == ["cast_multi"] + gemms
    assert rec.calls[0][1][0] == 4
    rec.calls = []
    block.step(x[0], None, None, x[3], stream=0)
    assert rec.names() == ["cast_multi"] + gemms and rec.calls[0][1][0] == 2
    rec.calls = []
    block.forward(x[0], stream=0)
    block.backward(x[3], stream=0)
    block.backward(x[3], stream=0, cast_g=False)
    cast = "cast_fp8" if operand == "fp8" else "residual_add"
    assert rec.names() == [cast] + apart[:2] + [cast] + apart[2:] + apart[2:]


def test_a_refused_group_adds_the_bias_in_single_launches(monkeypatch):
    class Refuses(_Recorder):
        def __getattr__(self, name):
            call = super().__getattr__(name)
            return (lambda *args: call(*args) or L.US_ERR_UNSUPPORTED) if name == "us_linear_group_bias" else call
    block, x = _ffn()
    rec = Refuses()
    monkeypatch.setattr(L, "_lib", rec)
    block.step(*x, stream=0)
    assert rec.names()[3:] == ["linear_group_bias", "linear_bwd_w", "linear_bwd_w", "linear_fwd_bias", "linear_bwd_x"]
    assert rec.calls[6][1][3].ptr == block.b2.data_ptr()


def test_a_copy_has_its_own_buffers(monkeypatch):
    block, x = _ffn()
    rec = _Recorder()
    monkeypatch.setattr(L, "_lib", rec)
    block.step(*x, stream=0)
    other = copy.deepcopy(block)
    rec.calls = []
    other.step(*x, stream=0)
    mine = {t.data_ptr() for t in block._owned()}
    assert not mine & {a._obj.ptr for _, args in rec.calls for a in args if isinstance(getattr(a, "_obj", None), L.us_mat)}


def test_a_changed_bias_buffer_lays_the_step_out_anew(monkeypatch):
    block, x = _ffn()
    rec = _Recorder()
    monkeypatch.setattr(L, "_lib", rec)
    block.step(*x, stream=0)
    block.b1 = torch.ones(48)
    rec.calls = []
    block.step(*x, stream=0)
    assert rec.calls[1][1][3]._obj.ptr == block.b1.data_ptr()


def test_arguments_that_do_not_fit():
    block, x = _ffn()
    with pytest.raises(ValueError):
        block.step(x[0], x[1], None, x[3])
    with pytest.raises(NotImplementedError):
        block.stages()
    p, g = torch.zeros(4, 4), torch.zeros(4, 4)
    for bad in (dict(params=[p], grads=[]), dict(params=[p], grads=[g[:2]]), dict(params=[], grads=[]), dict(params=[p.half()], grads=[g]), dict(params=[p], grads=[g], states="4bit"),
                dict(params=[p], grads=[g], copies=[None, None]), dict(params=[p], grads=[g], weight_decay=[0.0, 0.0])):
        with pytest.raises(ValueError):
            optim.AdamW(**bad)
