"""us_linear_fwd_bias against the oracle, in every tiling of the linear ops and with every epilogue.

Tolerances as for the linear ops: float32 results within TOL = 2e-3 (unit-scale products, of which the bias, added in the same fused multiply-add, is no part), 16-bit
ones one step more, FP8 codes one step.  An activation's slope times its factor is below 2 for all of them but sigmoid's 4.8 / 4 and tanh's 1.6.  Where the product is zero
the result is the bias, to the bit."""
import math

import pytest
import torch

from oracle import scales as S
from tests import util as U
from tests.test_gpu_linear_narrow import PAD, TOL

pytestmark = pytest.mark.gpu

# rows, contraction, columns: narrow tiles, 128 x 128, pairs (one and two tiles to a pair), and contractions shared by CTAs and by pairs; columns that end
# inside a slice of 32
TILES = [(1, 16, 16), (1, 1024, 4096), (40, 144, 33), (129, 272, 81), (200, 80, 4700), (9400, 80, 80), (1000, 400, 1040), (2600, 80, 1063), (4096, 96, 1537),
         (48, 4096, 1024), (300, 5008, 690), (2048, 6400, 1024)]
BIASES = ["f32", "bf16", "fp16"]
# mantissa bits, exponent of the smallest normal number, largest number
FORMATS = {"bf16": (7, -126, math.inf), "fp16": (10, -14, 65504.0), "e4m3": (3, -6, 448.0), "e5m2": (2, -14, 57344.0)}


def _lib():
    from paper_2303_11257_b200 import lib
    return lib


def _close(got, ref, fmt, tol, what=""):
    """got against 64-bit values: within tol, and one step of its format more."""
    got, off = got.double(), tol
    if fmt != "f32":
        mantissa, least, most = FORMATS[fmt]
        ref = ref.clamp(-most, most)
        off = tol + torch.ldexp(torch.ones_like(ref), (torch.frexp(ref.abs().clamp(min=2.0 ** least))[1] - 1 - mantissa))
    bad = ~((got - ref).abs() <= off)
    assert not bool(bad.any()), (what, int(bad.sum()), float((got - ref).abs().max()))


def _normal(rows, cols, fmt, seed):
    """A matrix of N(0, 1) with rows on 16-byte boundaries, and its values in 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(1000 * seed + rows + cols)
    t = U.empty(rows, cols, fmt, PAD(cols))
    t.copy_(torch.randn((rows, cols), generator=gen, device="cuda"))
    return t, t.double()


def _make(shape, fmt, bias_fmt):
    b, m, n = shape
    (X, x), (W, w) = _normal(b, m, fmt, 1), _normal(m, n, fmt, 2)
    bias = torch.zeros((1, n + 1), dtype=U.TORCH_OF[bias_fmt], device="cuda")[:, 1:]          # an element behind a boundary
    bias.copy_(_normal(1, n, "f32", 3)[0] + (0.01 * torch.arange(n, device="cuda")) % 3)
    return (X, W, bias), (x @ w) * float(torch.tensor(m ** -0.5)) + bias.double()


def _tol(val):
    return TOL * max(1.0, float(val.abs().max()) / 4)


def _act(name, z):
    return {"gelu": lambda: z * torch.special.ndtr(z), "relu": lambda: z.clamp(min=0), "tanh": lambda: torch.tanh(z), "sigmoid": lambda: torch.sigmoid(z)}[name]()


def _call(n, out, L, *args, **kw):
    """The call, and that nothing is written behind the 16 bytes in which a row ends."""
    ws = L.new_workspace()
    L.us_linear_fwd_bias(*args, ws, **kw)
    assert L.us_workspace_status(ws) == 0
    for t in (out, kw.get("Yq")):
        if t is not None and t.shape[0] > 1:
            whole = t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1)).contiguous().view(torch.uint8)
            assert not whole[:, -(-n * t.element_size() // 16) * 16:].any()


@pytest.mark.parametrize("shape", TILES)
@pytest.mark.parametrize("fmt,out", [("e4m3", "f32"), ("e4m3", "e4m3"), ("e4m3", "e5m2"), ("e4m3", "bf16"), ("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "f32"), ("fp16", "e4m3")])
def test_plain(shape, fmt, out):
    L = _lib()
    (X, W, bias), val = _make(shape, fmt, BIASES[(shape[0] + len(out)) % 3])
    Y = U.empty(shape[0], shape[2], out, PAD(shape[2]))
    _call(shape[2], Y, L, X, W, shape[1] ** -0.5, bias, Y)
    _close(Y, val, out, _tol(val), f"{shape} {fmt} {out}")


@pytest.mark.parametrize("shape", TILES)
@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
@pytest.mark.parametrize("bias_fmt", BIASES)
def test_a_product_of_zero_leaves_the_bias(shape, fmt, bias_fmt):
    L = _lib()
    (X, W, bias), _ = _make(shape, fmt, bias_fmt)
    X.copy_(torch.zeros_like(X, dtype=torch.float32))
    n, ws = shape[2], L.new_workspace()
    for out in ("f32", "bf16", "e4m3"):
        Y = U.empty(shape[0], n, out, PAD(n))
        L.us_linear_fwd_bias(X, W, 1.0, bias[0], Y, ws)
        want = bias.float().clamp(-448, 448).to(Y.dtype) if out == "e4m3" else bias.float().to(Y.dtype)
        assert torch.equal(Y.float(), want.float().expand(shape[0], n)), (shape, out)
    H, Y = U.empty(shape[0], n, "bf16", PAD(n)), U.empty(shape[0], n, "e4m3", PAD(n))
    L.us_linear_fwd_bias(X, W, 1.0, bias[0], Y, ws, L.epilogue(act=L.US_ACT_GELU, aux=H))
    assert torch.equal(H.float(), bias.float().to(torch.bfloat16).float().expand(shape[0], n))
    skip = torch.randn((shape[0], n), device="cuda")
    sk = torch.zeros((shape[0], PAD(n)), device="cuda")[:, :n].copy_(skip)
    Y = U.empty(shape[0], n, "f32", PAD(n))
    L.us_linear_fwd_bias(X, W, 1.0, bias[0], Y, ws, L.epilogue(skip=sk, skip_coef=1.0, out_coef=0.5))
    assert torch.equal(Y, skip + 0.5 * bias.float())
    assert L.us_workspace_status(ws) == 0


@pytest.mark.parametrize("shape", TILES)
@pytest.mark.parametrize("act", ["gelu", "relu", "tanh", "sigmoid"])
@pytest.mark.parametrize("fmt,out,aux", [("e4m3", "e4m3", "bf16"), ("e4m3", "e5m2", None), ("e4m3", "f32", "fp16"), ("bf16", "bf16", "bf16"), ("fp16", "fp16", None)])
def test_activations(shape, act, fmt, out, aux):
    L = _lib()
    b, m, n = shape
    (X, W, bias), val = _make(shape, fmt, BIASES[(b + len(act)) % 3])
    Y, H = U.empty(b, n, out, PAD(n)), U.empty(b, n, aux, PAD(n)) if aux else None
    f = float(getattr(S, act + "_scales")()[0])
    ep = L.epilogue(act=getattr(L, "US_ACT_" + act.upper()), act_in_scale=0.9, act_out_scale=f, aux=H)
    _call(n, Y, L, X, W, m ** -0.5, bias, Y, ep=ep)
    tol = _tol(val)
    if H is not None:
        _close(H, val, aux, tol, "kept")
    _close(Y, f * _act(act, 0.9 * val), out, 2 * tol, f"{shape} {act} {out}")


@pytest.mark.parametrize("shape", TILES)
@pytest.mark.parametrize("fmt,out,skip", [("e4m3", "bf16", "f32"), ("e4m3", "f32", "bf16"), ("bf16", "bf16", "bf16"), ("fp16", "fp16", "f32"), ("e4m3", "e4m3", "fp16")])
def test_residuals_and_their_copies(shape, fmt, out, skip):
    L = _lib()
    b, m, n = shape
    (X, W, bias), val = _make(shape, fmt, BIASES[b % 3])
    sk, skv = _normal(b, n, skip, 4)
    Y, ep = U.empty(b, n, out, PAD(n)), L.epilogue(skip=sk, skip_coef=0.8, out_coef=0.6)
    tol = _tol(val)
    _call(n, Y, L, X, W, m ** -0.5, bias, Y, ep=ep)
    _close(Y, 0.8 * skv + 0.6 * val, out, tol, f"{shape} residual")
    if out != "e4m3":
        Z, q = U.empty(b, n, out, PAD(n)), U.empty(b, n, "e4m3", PAD(n))
        _call(n, Z, L, X, W, m ** -0.5, bias, Z, ep=ep, Yq=q)
        assert torch.equal(Z.contiguous().view(torch.uint8), Y.contiguous().view(torch.uint8))
        assert torch.equal(q.float(), Y.float().clamp(-448, 448).to(torch.float8_e4m3fn).float())


@pytest.mark.parametrize("shape", TILES)
@pytest.mark.parametrize("act", ["gelu", "tanh"])
@pytest.mark.parametrize("fmt,out,aux,skip", [("e4m3", "bf16", "bf16", "f32"), ("bf16", "bf16", None, "bf16"), ("e4m3", "e4m3", None, "fp16"), ("fp16", "fp16", "fp16", "f32"),
                                              ("e4m3", "f32", None, "f32")])
def test_activation_and_residual_together(shape, act, fmt, out, aux, skip):
    L = _lib()
    b, m, n = shape
    (X, W, bias), val = _make(shape, fmt, BIASES[b % 3])
    sk, skv = _normal(b, n, skip, 4)
    Y, H = U.empty(b, n, out, PAD(n)), U.empty(b, n, aux, PAD(n)) if aux else None
    f = float(getattr(S, act + "_scales")()[0])
    ep = L.epilogue(act=getattr(L, "US_ACT_" + act.upper()), act_in_scale=0.9, act_out_scale=f, aux=H, skip=sk, skip_coef=0.8, out_coef=0.6)
    _call(n, Y, L, X, W, m ** -0.5, bias, Y, ep=ep)
    tol = _tol(val)
    if H is not None:
        _close(H, val, aux, tol, "kept")
    _close(Y, 0.8 * skv + 0.6 * f * _act(act, 0.9 * val), out, 2 * tol, f"{shape} {act} and residual")


@pytest.mark.parametrize("shape", [(1, 1024, 4096), (1000, 400, 1040), (2600, 80, 1063), (48, 4096, 1024)])
@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
def test_a_bias_of_zero_changes_nothing(shape, fmt):
    """To the bit what us_linear_fwd gives."""
    L = _lib()
    b, m, n = shape
    (X, W, bias), _ = _make(shape, fmt, "f32")
    zero, ws = torch.zeros(n, device="cuda"), L.new_workspace()
    for out in ("f32", "bf16", "e4m3"):
        for ep in (None, L.epilogue(act=L.US_ACT_GELU, act_out_scale=1.7), L.epilogue(skip=torch.randn((b, PAD(n)), device="cuda")[:, :n], skip_coef=0.8, out_coef=0.6)):
            Y, Z = U.empty(b, n, out, PAD(n)), U.empty(b, n, out, PAD(n))
            L.us_linear_fwd(X, W, m ** -0.5, Y, ws, ep)
            L.us_linear_fwd_bias(X, W, m ** -0.5, zero, Z, ws, ep)
            assert torch.equal(Y.float(), Z.float())


def test_nan_and_infinity_of_a_bias():
    L = _lib()
    (X, W, bias), val = _make((300, 80, 500), "bf16", "f32")
    bias[0, 3], bias[0, 499] = float("nan"), float("inf")
    Y = U.empty(300, 500, "f32", 512)
    L.us_linear_fwd_bias(X, W, 80 ** -0.5, bias, Y, L.new_workspace())
    assert bool(torch.isnan(Y[:, 3]).all()) and bool(torch.isinf(Y[:, 499]).all()) and bool(torch.isfinite(Y[:, 4:499]).all())


def test_captured_with_a_bias_that_changes():
    """The bias is read when the launch runs: a replay after an update of it in the same graph."""
    L = _lib()
    (X, W, bias), _ = _make((512, 128, 640), "e4m3", "f32")
    Y, ws = U.empty(512, 640, "f32"), L.new_workspace()
    b = bias[0].clone()
    p, g = b, torch.ones(640, device="cuda")
    plan, step = L.adamw_tensors([p], [g], [torch.zeros(640, device="cuda")], [torch.zeros(640, device="cuda")]), L.new_adamw_step()
    L.us_linear_fwd_bias(X, W, 0.1, b, Y, ws)
    before = Y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.us_adamw(plan, step, 0.25)
        L.us_linear_fwd_bias(X, W, 0.1, b, Y, ws)
    for i in range(1, 5):
        graph.replay()
        assert float((before - 0.25 * i - Y).abs().max()) < 1e-4, i


@pytest.mark.parametrize("rows,n", [(3, 2049), (300, 2049)])
@pytest.mark.parametrize("act", ["relu", "tanh", "sigmoid"])
@pytest.mark.parametrize("skip", [False, True])
def test_activations_over_their_range(rows, n, act, skip):
    """Products of zero, so that the activation's argument is in_scale * bias: from -100 to 100, small ones, infinities and NaN.  Sigmoid: e^-z errs by 2^-22 and, as z log2 e is
    rounded, by |z| 2^-23 log2 e, the reciprocal by 2^-23, sum and factor by 2^-24 each.  Tanh is 2 s - 1, absolute, from 1/8 on, and below that a series whose next term
    is 2^-22 of it, with four roundings."""
    L = _lib()
    z = torch.cat([torch.linspace(-100, 100, n // 2), 0.13 * torch.linspace(-1, 1, n - n // 2 - 8), torch.tensor([0.0, -0.0, 1e-20, -1e-20, 0.125, float("inf"), float("-inf"), float("nan")])])
    X, W = torch.zeros((rows, 64), device="cuda").bfloat16(), torch.zeros((64, PAD(n)), device="cuda").bfloat16()[:, :n]
    Y, S = U.empty(rows, n, "f32", PAD(n)), torch.zeros((rows, PAD(n)), device="cuda")[:, :n]
    code = {"relu": L.US_ACT_RELU, "tanh": L.US_ACT_TANH, "sigmoid": L.US_ACT_SIGMOID}[act]
    ep = L.epilogue(act=code, act_in_scale=0.5, act_out_scale=1.5, skip=S if skip else None, skip_coef=0.5 if skip else 0.0, out_coef=1.0)
    _call(n, Y, L, X, W, 1.0, (2.0 * z).cuda(), Y, ep=ep)
    ref, zz = 1.5 * _act(act, z.double()), z.double().abs()
    got = Y[-1].cpu().double()
    assert bool((Y == Y[0]).logical_or(Y.isnan()).all()) and bool(got[-1].isnan()) and bool(got[:-1].isfinite().all()) == (act != "relu")
    tol = {"relu": 2.0 ** -23 * ref.abs(), "sigmoid": (2.0 ** -20 + zz * 2.0 ** -22) * ref.abs() + 2.0 ** -125,
           "tanh": torch.where(zz < 0.125, 2.0 ** -21 * ref.abs(), 2.0 ** -19 * torch.ones_like(zz))}[act]
    keep = torch.isfinite(z)
    assert bool(((got - ref).abs() <= tol)[keep].all()), float(((got - ref).abs() / tol)[keep].nan_to_num().max())
    assert torch.equal(got[[-3, -2]], ref[[-3, -2]])
