"""What a gated FFN block and an encoder layer with norms of queries and keys issue, without a GPU: the calls and their order, copies of
a block, arguments that have to fit."""
import copy

import pytest
import torch

from paper_2303_11257_b200 import encoder, ffn
from paper_2303_11257_b200 import lib as L


class _Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return L.US_OK
        return call

    def names(self):
        return [n[3:] for n, _ in self.calls]


def _ffn(**kw):
    return ffn.UnitScaledGatedFFN(64, 32, 48, device="cpu", **kw), [torch.zeros(s) for s in ((64, 32), (32, 96), (48, 32), (64, 32))]


def _layer(**kw):
    kw = {"fused_attention": True, "gate": "silu", **kw}
    w = 512 if kw["gate"] else 256
    x = [torch.zeros(s) for s in ((128, 128), (128, 384), (128, 128), (128, w), (256, 128), (128, 128))]
    return encoder.UnitScaledEncoderLayer(2, 64, 128, 2, 256, device="cpu", **kw), x


def test_a_step_of_the_block_is_four_calls(monkeypatch):
    block, x = _ffn()
    rec = _Recorder()
    monkeypatch.setattr(L, "_lib", rec)
    block.step(*x, stream=0)
    assert rec.names() == ["cast_multi", "ffn_gated_fwd", "ffn_gated_bwd", "linear_group_any"]
    rec.calls = []
    block.forward(x[0], stream=0)
    block.backward(x[3], stream=0)
    block.backward(x[3], stream=0, cast_g=False)
    assert rec.names() == ["cast_fp8", "ffn_gated_fwd", "linear_fwd", "cast_fp8", "ffn_gated_bwd", "linear_group_any", "ffn_gated_bwd", "linear_group_any"]


def test_a_copy_has_its_own_buffers(monkeypatch):
    block, x = _ffn(operand="bf16", kept="e4m3")
    rec = _Recorder()
    monkeypatch.setattr(L, "_lib", rec)
    block.step(*x, stream=0)
    other = copy.deepcopy(block)
    rec.calls = []
    other.step(*x, stream=0)
    mine = {t.data_ptr() for t in block._owned()}
    assert not mine & {a._obj.ptr for _, args in rec.calls for a in args if isinstance(getattr(a, "_obj", None), L.us_mat)}


@pytest.mark.parametrize("attention,fused", [("bf16", True), ("fp8", True), ("fp16", False), ("fp8", False)])
def test_norms_of_queries_and_keys_stand_around_attention(attention, fused, monkeypatch):
    monkeypatch.setattr(L, "rotary_table", lambda n, r, base, device: torch.zeros(n, r))          # (made by a kernel)
    layer, x = _layer(attention=attention, fused_attention=fused, qk_norm=True, rotary=10000.0)
    rec = _Recorder()
    monkeypatch.setattr(L, "_lib", rec)
    layer.step(*x, stream=0, qk=[torch.ones(64)] * 2)
    n = rec.names()
    assert n.count("qk_norm_fwd") == n.count("qk_norm_bwd") == n.count("ffn_gated_fwd") == n.count("ffn_gated_bwd") == 1
    i, j = n.index("qk_norm_fwd"), n.index("qk_norm_bwd")
    assert n[i - 1] == "linear_fwd" and (n[i + 1] == "cast_fp8") == (attention == "fp8") and n[j + 1] == "linear_group_any" and j == len(n) - 2
    between = n[i + 1:j]
    assert any(c.startswith("attention_fwd" if fused else "softmax_fwd") for c in between) and any(c.startswith("attention_bwd" if fused else "softmax_bwd") for c in between)


def test_what_does_not_fit_is_refused():
    with pytest.raises(ValueError):
        ffn.UnitScaledGatedFFN(64, 32, 40, device="cpu")
    with pytest.raises(ValueError):
        ffn.UnitScaledGatedFFN(64, 32, 48, gate="swish", device="cpu")
    with pytest.raises(AssertionError):
        encoder.UnitScaledEncoderLayer(2, 64, 128, 2, 256, device="cpu", rotary=10000.0)
    with pytest.raises(NotImplementedError):
        _ffn()[0].stages(None, None, None, None)


def test_factors():
    sc = ffn.GatedScales.unit(64, 32, 48, "gelu")
    assert abs(sc.alpha1 - 32 ** -0.5) < 1e-7 and abs(sc.beta_x1 - 96 ** -0.5) < 1e-7 and abs(sc.beta_w - 64 ** -0.5) < 1e-7 and abs(sc.alpha2 - 48 ** -0.5) < 1e-7
    assert (sc.alpha_g, sc.beta_h, sc.beta_u) == L.us_scales_gated("gelu")
    c = ffn.GatedScales.unit(64, 32, 48, "gelu", constrained=True)
    assert c.alpha1 == c.beta_x1 and c.alpha_g == c.beta_h == c.beta_u and c.alpha2 == c.beta_x2
    assert abs(ffn.GatedScales.unit(64, 32, 48, dp_world=4).beta_w - 256 ** -0.5) < 1e-7


def test_a_changed_factor_of_the_norms_weights_is_used(monkeypatch):
    """beta_qk belongs to what a step was laid out for, as beta_ln does."""
    layer, x = _layer(qk_norm=True, norm="post")
    rec = _Recorder()
    monkeypatch.setattr(L, "_lib", rec)
    ln = [torch.ones(128)] * 4

    def factors():
        rec.calls = []
        layer.step(*x, stream=0, qk=[torch.ones(64)] * 2, ln=ln)
        (args,) = [a for n, a in rec.calls if n == "us_qk_norm_bwd"]
        return [float(v) for v in args[6]], {float(a[5]) for n, a in rec.calls if n == "us_layer_norm_bwd_cast"}
    first, _ = factors()
    assert first == [layer.beta_qk] * 2
    layer.beta_qk = 0.25
    assert factors() == ([0.25, 0.25], {layer.beta_ln})
    layer.beta_ln = 0.125
    assert factors() == ([0.25, 0.25], {0.125})
