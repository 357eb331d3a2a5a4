"""Forms of the gated FFN kernels and of a layer with norms of queries and keys that only some sizes take: bands of several tile rows (weights beyond
what stays in L2), wide tiles of single CTAs over few rows with one and several tiles a CTA, results beyond 2^31 elements, and the
backward pass of fused attention in three launches between the norms' two.  Tolerances as in test_gpu_ffn_gated; where contractions are long their sums are exact."""
import numpy as np
import pytest
import torch

from oracle import encoder as E
from oracle import ops as O
from tests import util as U
from tests.test_gpu_ffn_gated import _backward, _close, _forward, _pitch
from tests.test_gpu_gated_block import _host, _near

pytestmark = pytest.mark.gpu


def _lib():
    from paper_2303_11257_b200 import lib
    return lib


def _on_device(gen, r, c, fmt):
    t = U.empty(r, c, fmt, _pitch(c))
    return t.copy_(torch.randn((r, c), generator=gen, device="cuda"))


def _rows(b):
    """Both ends of every tile row of 128 (the last ragged), and some between."""
    at = np.arange(0, b, 128)
    return np.unique(np.concatenate([at, at + 127, at + 61, [b - 1]]).clip(0, b - 1))


def _signs(gen, r, c, fmt):
    """-1, 0 and 1, whose sums of products are whole numbers far below 2^24: exact in float32, in any order."""
    t = U.empty(r, c, fmt, _pitch(c))
    return t.copy_(torch.randint(-1, 2, (r, c), generator=gen, device="cuda").float())


def _product(a, w, scale):
    """scale * a w for such operands, and what the multiplication by scale may be off by."""
    v = (np.float64(np.float32(scale)) * (a.double() @ w.double())).cpu().numpy()
    return v, 2.0 ** -24 * np.abs(v)


# Weights of more than 64 MB.  CTA pairs, six tile rows in bands of four: lanes' stores.  Narrow tiles, nine tile rows in bands of eight, a very long contraction.
BANDS = {"pairs16": (1300, 2064, 8200, "bf16", "bf16", "bf16"), "pairs8": (1300, 4112, 8200, "e4m3", "e5m2", "e4m3"), "narrow": (1100, 250000, 70, "fp16", "fp16", "fp16")}


@pytest.mark.parametrize("case", BANDS)
def test_forward_in_bands(case):
    b, m, f, fmt, _, kept = BANDS[case]
    L, gen = _lib(), torch.Generator(device="cuda").manual_seed(3)
    X, Wg, Wu = _signs(gen, b, m, fmt), _signs(gen, m, f, fmt), _signs(gen, m, f, fmt)
    A, H, V = U.empty(b, f, fmt, _pitch(f)), U.empty(b, f, kept, _pitch(f)), U.empty(b, f, kept, _pitch(f))
    ws = L.new_workspace()
    L.us_ffn_gated_fwd("silu", X, Wg, Wu, m ** -0.5, A, ws, H=H, U=V, act_out_scale=1.625)
    assert L.us_workspace_status(ws) == 0
    at = torch.from_numpy(_rows(b)).cuda()
    pick = lambda t: (t.view(torch.uint8)[at].view(t.dtype) if t.element_size() == 1 else t[at])
    x = pick(X).float()
    (h, eh), (u, eu) = _product(x, Wg.float(), m ** -0.5), _product(x, Wu.float(), m ** -0.5)
    fv = np.abs(O.activation_fwd("silu", h, 1.0, 1.0))
    _close(pick(H), h, eh, kept, "H")
    _close(pick(V), u, eu, kept, "U")
    _close(pick(A), O.activation_fwd("silu", h, 1.0, 1.625) * u, 1.625 * (1.13 * eh * np.abs(u) + fv * eu + (3e-6 * fv + 1e-6) * np.abs(u)), fmt, "A")


@pytest.mark.parametrize("case", BANDS)
def test_backward_in_bands(case):
    b, n, f, act, grad, kept = BANDS[case]
    n *= 2                                                       # one weight, not two
    L, gen = _lib(), torch.Generator(device="cuda").manual_seed(4)
    G, W2, H, V = _signs(gen, b, n, grad), _signs(gen, f, n, act), _on_device(gen, b, f, kept), _on_device(gen, b, f, kept)
    dH, dU, ws = U.empty(b, f, grad, _pitch(f)), U.empty(b, f, grad, _pitch(f)), L.new_workspace()
    L.us_ffn_gated_bwd("silu", G, W2, n ** -0.5, H, V, dH, dU, ws, beta_h=1.5, beta_u=1.25)
    assert L.us_workspace_status(ws) == 0
    at = torch.from_numpy(_rows(b)).cuda()
    pick = lambda t: (t.view(torch.uint8)[at].view(t.dtype) if t.element_size() == 1 else t[at])
    d, e = _product(pick(G).float(), W2.float().t(), n ** -0.5)
    h, u = U.host_values(pick(H)), U.host_values(pick(V))
    fv, df = O.activation_fwd("silu", h, 1.0, 1.0), O.activation_bwd("silu", h, np.ones_like(h), 1.0, 1.0)
    _close(pick(dU), 1.25 * fv * d, 1.25 * (np.abs(fv) * e + (3e-6 * np.abs(fv) + 1e-6) * np.abs(d)), grad, "dU")
    _close(pick(dH), 1.5 * df * u * d, 1.5 * np.abs(u) * (np.abs(df) * e + (3e-6 * np.abs(df) + 2e-6) * np.abs(d)), grad, "dH")


@pytest.mark.parametrize("b,f", [(37, 5000), (37, 20000), (128, 10000), (1, 20008)])
@pytest.mark.parametrize("fmt,grad,kept", [("bf16", "bf16", "bf16"), ("e4m3", "e5m2", "e4m3"), ("e4m3", "e5m2", "bf16")])
def test_wide_tiles_over_few_rows(b, f, fmt, grad, kept):
    """More hidden columns than the machine has narrow tiles for: 4736 forward and 9472 backward on 148 SMs; several tiles a CTA from 9472 and 18944 on."""
    _forward((b, 80, f, 0), "silu", fmt, kept)
    _backward((b, 0, f, 96), "silu", fmt, grad, kept)


@pytest.mark.parametrize("m", [272, 1168])
def test_results_beyond_32_bits(m):
    """Rows 1.6 million elements apart, all five results (and the copies that the backward pass reads) in one buffer, whose last row starts 4.6e9 elements in: the bits
    of the same call on matrices of their own.  Contractions of both lengths: results leave by TMA and by the lanes' stores."""
    L = _lib()
    b, f, n, pitch = 2900, 1808, 64, 1_600_000
    gen = torch.Generator(device="cuda").manual_seed(5)
    X, Wg, Wu, G, W2 = (_on_device(gen, r, c, "bf16") for r, c in ((b, m), (m, f), (m, f), (b, n), (f, n)))
    buf = torch.empty(b * pitch, dtype=torch.bfloat16, device="cuda")
    far = [torch.as_strided(buf, (b, f), (pitch, 1), 2048 * i) for i in range(5)]
    near, ws = [torch.empty(b, f, dtype=torch.bfloat16, device="cuda") for _ in range(5)], L.new_workspace()
    for A, H, V, dH, dU in (near, far):
        L.us_ffn_gated_fwd("silu", X, Wg, Wu, m ** -0.5, A, ws, H=H, U=V)
        L.us_ffn_gated_bwd("silu", G, W2, n ** -0.5, H, V, dH, dU, ws)
    assert L.us_workspace_status(ws) == 0
    assert all(torch.equal(a, b) for a, b in zip(near, far))
    del buf, far


@pytest.mark.parametrize("attention,norm,gate,rotary", [("bf16", None, "silu", 10000.0), ("fp8", "post", "silu", 10000.0), ("fp16", "post", None, None)])
def test_layer_with_norms_and_attention_gradients_in_three_launches(attention, norm, gate, rotary):
    """144 keys of 9 problems: dQ and dK go to the norms' own gradients, dV to the projection's, on two streams."""
    from paper_2303_11257_b200 import encoder
    nseq, slen, d, nhead, f = 3, 144, 192, 3, 400
    T, w = nseq * slen, f * (2 if gate else 1)
    host = _host(71, (T, d), (d, 3 * d), (d, d), (d, w), (f, d), (T, d))
    more = _host(72, (1, d), (1, d), (1, d), (1, d), (1, 64), (1, 64))
    ln = [np.float32(v[0] * 0.2 + (1 - i % 2)) for i, v in enumerate(more[:4])] if norm else None
    qk = [np.float32(1 + 0.2 * v[0]) for v in more[4:]]
    cuda = lambda ts: None if ts is None else [torch.from_numpy(t).cuda() for t in ts]
    layer = encoder.UnitScaledEncoderLayer(nseq, slen, d, nhead, f, attention=attention, fused_attention=True, norm=norm, gate=gate, qk_norm=True, rotary=rotary)
    assert not layer.whole_bwd
    x, n, k = cuda(host), cuda(ln), cuda(qk)
    for _ in range(2):                                           # laid out, and as a program
        layer.step(*x, ln=n, qk=k)
        layer.check()
    r = E.encoder_layer(*host, nseq, slen, nhead, att=attention, norm=norm, ln=ln, fused_scores=True, gate=gate, qk=qk, rotary=rotary)
    tol = 8e-2 if attention == "fp8" else 5e-2
    for name, got, ref in (("QKn", layer.QKn, r.QKn), ("P", layer.P, r.P), ("R1", layer.R1, r.R1)):
        _near(got, ref, name, 2e-2, 0.995)
    for name, got, ref in (("dQKn", layer.dQKn, r.dQKn), ("dQKV", layer.dQKV, r.dQKV), ("dX", layer.dX, r.dX), ("dWqkv", layer.dWqkv, r.dWqkv), ("dWo", layer.dWo, r.dWo),
                           ("dW1", layer.ffn.dW1, r.ffn.dW1), ("dwq", layer.dqk[0], r.dqk[0]), ("dwk", layer.dqk[1], r.dqk[1])):
        _near(got, ref, name, tol, 0.99)
    outs = (layer.dX, layer.dQKn, layer.dQKVq, layer.dWqkv, layer.ffn.dW1, *layer.dqk)
    raw = lambda: [(t.view(torch.uint8) if t.element_size() == 1 else t).clone() for t in outs]
    want = raw()
    layer.step(*x, ln=n, qk=k, stream=torch.cuda.current_stream())               # one stream
    layer.check()
    assert all(torch.equal(a, b) for a, b in zip(want, raw()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(*x, ln=n, qk=k)
    graph.replay()
    layer.check()
    assert all(torch.equal(a, b) for a, b in zip(want, raw()))
