"""The gated FFN block and encoder layers with a gated block and norms of queries and keys: a run of the operators together, against
the oracle's chain.  Each operator is checked strictly on its own; here tensors early in the chain are held to a step of their format and later
ones statistically, as for the plain block and layer: a code that rounds the other way moves all that follows."""
import numpy as np
import pytest
import torch

from oracle import encoder as E
from oracle import ops as O
from tests import util as U

pytestmark = pytest.mark.gpu


def _host(seed, *shapes):
    from paper_2303_11257_b200 import synth
    return [synth.normal(seed, i, s) for i, s in enumerate(shapes)]


def _near(got, ref, name, mean_tol=1e-2, corr=0.999):
    g, scale = U.host_values(got), max(1e-6, float(np.abs(ref).std()))
    err = np.abs(g - ref) / scale
    assert err.mean() <= mean_tol, f"{name}: mean err {err.mean():.3e}"
    assert np.corrcoef(g.ravel(), ref.ravel())[0, 1] > corr, name


@pytest.mark.parametrize("T,d,f", [(96, 64, 80), (300, 144, 400), (1024, 272, 1104)])
@pytest.mark.parametrize("operand,kept,gate", [("fp8", "bf16", "silu"), ("fp8", "e4m3", "silu"), ("bf16", "bf16", "gelu"), ("fp16", "e4m3", "sigmoid")])
def test_block_against_the_oracle(T, d, f, operand, kept, gate):
    from paper_2303_11257_b200 import ffn
    X, W1, W2, G = _host(51, (T, d), (d, 2 * f), (f, d), (T, d))
    dev = [torch.from_numpy(t).cuda() for t in (X, W1, W2, G)]
    block = ffn.UnitScaledGatedFFN(T, d, f, operand=operand, gate=gate, kept=kept)
    block.step(*dev)
    block.check()
    r = O.gated_ffn_block(X, W1, W2, G, gate, operand=operand, kept=kept)
    fp8 = operand == "fp8"
    U.assert_close_stored(block.HU, r.H, kept, 2e-3 * max(1.0, np.abs(r.H).max() / 4), "kept projections")
    for name, got, ref in (("A", block.Aq, r.Aq), ("dHU", block.dHUq, r.dHq), ("R", block.R, r.R), ("dW2", block.dW2, r.dW2), ("dW1", block.dW1, r.dW1), ("dX", block.dX, r.dX)):
        _near(got, ref, name, 1e-2 if fp8 else 4e-3)
    # unit scale: A is the product's, dX and the weight gradients carry both halves
    assert 0.8 < float(np.std(r.dW1)) < 1.6
    # forward and backward on their own do what a step does
    want = [t.clone() for t in (block.R, block.dX, block.dW1, block.dW2)]
    block.cast_weights(dev[1], dev[2])
    block.forward(dev[0])
    block.backward(dev[3])
    assert all(torch.equal(a, b) for a, b in zip(want, (block.R, block.dX, block.dW1, block.dW2)))


@pytest.mark.parametrize("operand", ["fp8", "bf16"])
def test_captured_block_and_other_tensors(operand):
    from paper_2303_11257_b200 import ffn
    T, d, f = 256, 128, 512
    make = lambda seed: [torch.from_numpy(t).cuda() for t in _host(seed, (T, d), (d, 2 * f), (f, d), (T, d))]
    block, other, x, y = ffn.UnitScaledGatedFFN(T, d, f, operand=operand), ffn.UnitScaledGatedFFN(T, d, f, operand=operand), make(1), make(2)
    block.step(*x)
    torch.cuda.synchronize()
    graph = block.capture(*x)
    for a, b in zip(x, y):
        a.copy_(b)
    graph.replay()
    other.step(*[t.clone() for t in y], stream=torch.cuda.current_stream())
    block.check()
    other.check()
    assert all(torch.equal(a, b) for a, b in zip((block.R, block.dX, block.dW1, block.dW2), (other.R, other.dX, other.dW1, other.dW2)))
    assert block.launches_per_step == 1 + block.gemm_launches and block.gemm_launches >= 3


@pytest.mark.parametrize("attention,fused,norm,gate,rotary", [("bf16", True, None, "silu", 10000.0), ("fp8", True, "post", "silu", 10000.0), ("fp16", False, None, None, 500.0),
                                                              ("fp8", False, None, "gelu", None), ("bf16", True, "post", None, 10000.0)])
def test_layer_against_the_oracle(attention, fused, norm, gate, rotary):
    from paper_2303_11257_b200 import encoder
    nseq, slen, d, nhead, f = 3, 80, 192, 3, 400
    T, w = nseq * slen, f * (2 if gate else 1)
    host = _host(61, (T, d), (d, 3 * d), (d, d), (d, w), (f, d), (T, d))
    more = _host(62, (1, d), (1, d), (1, d), (1, d), (1, 64), (1, 64))
    ln = [np.float32(v[0] * 0.2 + (1 - i % 2)) for i, v in enumerate(more[:4])]
    qk = [np.float32(1 + 0.2 * v[0]) for v in more[4:]]
    cuda = lambda ts: [torch.from_numpy(t).cuda() for t in ts]
    layer = encoder.UnitScaledEncoderLayer(nseq, slen, d, nhead, f, attention=attention, fused_attention=fused, norm=norm, gate=gate, qk_norm=True, rotary=rotary)
    for _ in range(2):                                          # laid out, and as a program
        layer.step(*cuda(host), ln=cuda(ln) if norm else None, qk=cuda(qk))
        layer.check()
    r = E.encoder_layer(*host, nseq, slen, nhead, att=attention, norm=norm, ln=ln if norm else None, fused_scores=fused, gate=gate, qk=qk, rotary=rotary)
    wide = "bf16" if attention == "fp8" else attention
    U.assert_close_stored(layer.QKV, r.QKV, wide, 2e-3, "QKV")
    tol = 8e-2 if attention == "fp8" else 5e-2
    for name, got, ref in (("QKn", layer.QKn, r.QKn), ("P", layer.P, r.P), ("R1", layer.R1, r.R1)):
        _near(got, ref, name, 2e-2, 0.995)
    for name, got, ref in (("R", layer.R2 if norm else layer.ffn.R, r.R2 if norm else r.ffn.R), ("dQKn", layer.dQKn, r.dQKn), ("dQKV", layer.dQKV, r.dQKV), ("dX", layer.dX, r.dX),
                           ("dWqkv", layer.dWqkv, r.dWqkv), ("dWo", layer.dWo, r.dWo), ("dW1", layer.ffn.dW1, r.ffn.dW1), ("dW2", layer.ffn.dW2, r.ffn.dW2),
                           ("dwq", layer.dqk[0], r.dqk[0]), ("dwk", layer.dqk[1], r.dqk[1])):
        _near(got, ref, name, tol, 0.99)
    # the same step through a graph and with an explicit stream
    x, n, k = cuda(host), cuda(ln) if norm else None, cuda(qk)
    layer.step(*x, ln=n, qk=k)
    want = [t.clone() for t in (layer.dX, layer.dWqkv, layer.ffn.dW1, *layer.dqk)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(*x, ln=n, qk=k)
    for t in (layer.dX, layer.dWqkv, layer.ffn.dW1, *layer.dqk):
        t.zero_()
    graph.replay()
    layer.check()
    assert all(torch.equal(a, b) for a, b in zip(want, (layer.dX, layer.dWqkv, layer.ffn.dW1, *layer.dqk)))


@pytest.mark.parametrize("T,d,f,operand,kept", [(256, 128, 512, "fp8", "e4m3"), (16000, 128, 400, "fp8", "bf16"), (1000, 528, 2096, "bf16", "e4m3")])
def test_launches_of_a_gated_step(T, d, f, operand, kept):
    from paper_2303_11257_b200 import ffn
    from tests.test_gpu_launch_counts import _kernels
    block = ffn.UnitScaledGatedFFN(T, d, f, operand=operand, kept=kept)
    x = [torch.zeros(s, device="cuda") for s in ((T, d), (d, 2 * f), (f, d), (T, d))]
    assert _kernels(lambda: block.step(*x)) == block.launches_per_step


@pytest.mark.parametrize("attention,norm,fused,gate", [("bf16", None, True, "silu"), ("fp8", "post", True, "silu"), ("fp16", None, False, None), ("fp8", None, False, "gelu")])
def test_launches_of_a_layer_step(attention, norm, fused, gate):
    from paper_2303_11257_b200 import encoder
    from tests.test_gpu_launch_counts import _kernels
    nseq, slen, nhead = 4, 256, 2
    T, d, f = nseq * slen, 64 * nhead, 256 * nhead
    layer = encoder.UnitScaledEncoderLayer(nseq, slen, d, nhead, f, attention=attention, fused_attention=fused, norm=norm, gate=gate, qk_norm=True, rotary=10000.0)
    t = [torch.zeros(s, device="cuda") for s in ((T, d), (d, 3 * d), (d, d), (d, 2 * f if gate else f), (f, d), (T, d))]
    ln, qk = ([torch.ones(d, device="cuda") for _ in range(4)] if norm else None), [torch.ones(64, device="cuda") for _ in range(2)]
    assert _kernels(lambda: layer.step(*t, ln=ln, qk=qk)) == layer.kernel_launches
