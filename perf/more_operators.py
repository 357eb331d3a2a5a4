"""Operators that a training run with biases needs next to the scaled matmuls, as a list of measurable cases.

Kinds of work:
  linear_bias  matrix product with bias, activation and residual in its epilogue (`us_linear_fwd_bias`)
  bias_grad    gradients of the biases of an FFN block: column sums of the gradients of both layers' outputs (`us_bias_grad`)
  grad_norm    2-norm of the gradients of all tensors of a model, and the factor that clips them (`us_grad_norm`)
  adamw        an AdamW step over all tensors of a model at once, states in 32 or in 8 bits, with the next step's matmul
               operands (`us_adamw`)

With acc = X W:
  v = acc / sqrt(m) + b;  H = v in 16 bits;  v = alpha_g f(v);  Y = sqrt(1/2) skip + sqrt(1/2) v     (each part where the case has it)
  db = T^-1/2 sum over rows of G
  norm = sqrt(sum g^2),  factor = min(1, most / norm)
  g' = factor g;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2;
  p = (1 - lr wd) p - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps);  copy = p in the operands' format
States in 8 bits: in every block of 256 elements m = s_m c_m and sqrt(v) = s_v c_v with E4M3 codes c and s = (largest magnitude) / 448;
c_v is at least the smallest code where v > 0, so that no element loses its denominator.

Activations, gradients and weights are N(0, 1), the distribution unit scaling keeps them at.  `own` is false for the plain forms
below and true for the framework's kernels.
"""
import math

import torch

own = False

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": E4, "e5m2": E5}
MOST = {E4: 448.0, E5: 57344.0}
# 1 / std f(Z) for Z ~ N(0, 1)
FACTORS = {"gelu": 1.7009262, "relu": 1.7128585, "tanh": 1.5926870, "sigmoid": 4.8013}
HALF = math.sqrt(0.5)
BLOCK = 256
LR, BETAS, EPS, DECAY = 1e-3, (0.9, 0.999), 1e-8, 0.01


def _linear(tokens, m, n, operand, out, act="none", kept=False, skip="none", bias="f32"):
    """kept: the pre-activation is stored in BF16 (FP16 for FP16 operands) for the backward pass."""
    return {"kind": "linear_bias", "tokens": tokens, "m": m, "n": n, "operand": operand, "out": out, "act": act, "kept": kept, "skip": skip, "bias": bias}


def _grads(tokens, d, f, dtype):
    return {"kind": "bias_grad", "tokens": tokens, "d": d, "f": f, "dtype": dtype}


def _norm(layers, d, f, dtype):
    return {"kind": "grad_norm", "layers": layers, "d": d, "f": f, "dtype": dtype}


def _adamw(layers, d, f, states, grad="f32", copy="e4m3", steps=1000):
    """steps: made before this one."""
    return {"kind": "adamw", "layers": layers, "d": d, "f": f, "states": states, "grad": grad, "copy": copy, "steps": steps}


def listed():
    cases = {
        # one token of one sequence in evaluation, the first layer of a BERT-large FFN block: latency counts
        "linear_token": _linear(1, 1024, 4096, "bf16", "bf16", "gelu"),
        # a sub-batch left over at the end of an epoch, second layer of a block of pruned width: multiples of no tile
        "linear_ragged": _linear(1000, 2096, 528, "fp16", "fp16", skip="fp16", bias="fp16"),
        # the first and the second layer of the BERT-large block on 16 x 512 tokens in training, FP8
        "linear_bert_large_gelu": _linear(8192, 1024, 4096, "e4m3", "e4m3", "gelu", True),
        "linear_bert_large_residual": _linear(8192, 4096, 1024, "e4m3", "bf16", skip="f32"),
        # the projection of queries, keys and values at twice the width on twice the tokens: the largest product
        "linear_wide": _linear(16384, 2048, 6144, "bf16", "bf16"),
        # character language model (hidden 128, FFN 512, sequence 256): the smallest training step
        "bias_grad_char_lm": _grads(256, 128, 512, "bf16"),
        "bias_grad_bert_large": _grads(8192, 1024, 4096, "e5m2"),
        "norm_char_lm": _norm(4, 128, 512, "f32"),
        # the FFN blocks of all 24 layers of BERT-large
        "norm_bert_large": _norm(24, 1024, 4096, "f32"),
        "adamw_char_lm": _adamw(4, 128, 512, "f32", steps=0),
        "adamw_bert_large": _adamw(24, 1024, 4096, "f32"),
        # the same with states in 8 bits and gradients and operands in BF16
        "adamw_bert_large_8bit": _adamw(24, 1024, 4096, "8bit", "bf16", "bf16"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear_bias", "linear_bias", "bias_grad", "grad_norm", "adamw", "adamw"])
    while True:
        if kind == "linear_bias":
            operand = rng.choice(["e4m3", "e4m3", "bf16", "fp16"])
            wide = "bf16" if operand == "e4m3" else operand
            act = rng.choice(["none", "gelu", "gelu", "relu", "tanh", "sigmoid"])
            skip = rng.choice([wide, "f32"]) if act == "none" and rng.random() < 0.7 or rng.random() < 0.15 else "none"
            # (a layer of 16-bit operands hands on 16 bits)
            out = rng.choice(["bf16", "f32"] if skip != "none" else ["bf16", "e4m3", "f32"]) if operand == "e4m3" else operand
            c = _linear(_log(rng, 1, 16384), _log(rng, 64, 8192), _log(rng, 64, 8192), operand, out, act, act != "none" and rng.random() < 0.5, skip, rng.choice(["f32", wide]))
            if work(c)["flops"] <= 2.0 * 16384 * 2048 * 6144:
                return c
        elif kind == "bias_grad":
            c = _grads(_log(rng, 1, 16384), _log(rng, 64, 2048), _log(rng, 64, 8192), rng.choice(["e5m2", "bf16", "fp16", "f32"]))
            if work(c)["bytes"] <= 1 << 30:
                return c
        else:
            d = _log(rng, 64, 2048)
            size = (_log(rng, 1, 24), d, _log(rng, d, 8192))
            c = _norm(*size, rng.choice(["f32", "bf16", "fp16"])) if kind == "grad_norm" else \
                _adamw(*size, rng.choice(["f32", "8bit"]), rng.choice(["f32", "bf16"]), rng.choice(["e4m3", "bf16", "none"]), rng.choice([0, 0, _log(rng, 1, 100000)]))
            if size[0] * size[1] * size[2] <= 24 * 1024 * 4096:
                return c


def _padded(rows, cols, dtype):
    """A matrix with rows on 128-byte boundaries, as a matmul operand has them."""
    pitch = 128 // dtype.itemsize
    return torch.zeros((rows, -(-cols // pitch) * pitch), dtype=torch.uint8 if dtype.itemsize == 1 else dtype, device="cuda").view(dtype)[:, :cols]


def _normal(gen, m):
    return m.copy_(torch.randn(m.shape, generator=gen, device="cuda"))


def _shapes(case):
    """The tensors of a model of FFN blocks: all weights, then all biases."""
    n, d, f = case["layers"], case["d"], case["f"]
    return [s for _ in range(n) for s in ((d, f), (f, d))] + [s for _ in range(n) for s in ((f,), (d,))]


def _places(case):
    """Where each tensor begins in storage that holds all of them, each on a boundary of 256 elements, and the storage's size."""
    at, places = 0, []
    for s in _shapes(case):
        places.append(at)
        at += -(-math.prod(s) // BLOCK) * BLOCK
    return places, at


def _parts(flat, case):
    return [flat[i:i + math.prod(s)].view(s) for i, s in zip(_places(case)[0], _shapes(case))]


def _weights_end(case):
    """Where the biases begin in that storage."""
    places, _ = _places(case)
    return places[2 * case["layers"]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 31)
    s = {"case": case}
    if case["kind"] == "linear_bias":
        T, m, n, dt = case["tokens"], case["m"], case["n"], TYPES[case["operand"]]
        s["X"], s["W"] = _normal(gen, _padded(T, m, dt)), _normal(gen, _padded(m, n, dt))
        s["b"] = (0.5 * torch.randn((n,), generator=gen, device="cuda")).to(TYPES[case["bias"]])
        s["Y"] = _padded(T, n, TYPES[case["out"]])
        s["H"] = _padded(T, n, torch.float16 if case["operand"] == "fp16" else torch.bfloat16) if case["kept"] else None
        s["skip"] = _normal(gen, _padded(T, n, TYPES[case["skip"]])) if case["skip"] != "none" else None
        s["scratch"] = torch.zeros(4096, dtype=torch.uint8, device="cuda")
        return s
    if case["kind"] == "bias_grad":
        T, dt = case["tokens"], TYPES[case["dtype"]]
        s["G"] = [_normal(gen, _padded(T, w, dt)) for w in (case["f"], case["d"])]
        s["db"] = [torch.empty((w,), device="cuda") for w in (case["f"], case["d"])]
        return s
    _, size = _places(case)
    real = torch.zeros(size, device="cuda")                   # 1 where the storage holds an element of a tensor
    for p in _parts(real, case):
        p.fill_(1.0)
    if case["kind"] == "grad_norm":
        s["g"] = (torch.randn(size, generator=gen, device="cuda") * real).to(TYPES[case["dtype"]])
        s["out"], s["scratch"] = torch.zeros(2, device="cuda"), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
        return s
    # gradients whose size differs from element to element, and the moments that their past left
    sigma = torch.exp(torch.randn(size, generator=gen, device="cuda")) * real
    s["p"] = torch.randn(size, generator=gen, device="cuda") * real
    s["g"] = (sigma * torch.randn(size, generator=gen, device="cuda")).to(TYPES[case["grad"]])
    m, v = 0.3 * sigma * torch.randn(size, generator=gen, device="cuda"), sigma.square_()
    if case["steps"] == 0:
        m.zero_(), v.zero_()
    if case["states"] == "8bit":
        s["m"], s["m_scale"] = _codes(m)
        s["v"], s["v_scale"] = _codes(v.sqrt(), True)
    else:
        s["m"], s["v"] = m, v
    s["copies"] = [_padded(*t, TYPES[case["copy"]]) for t in _shapes(case)[:2 * case["layers"]]] if case["copy"] != "none" else []
    s["step"] = torch.tensor([case["steps"], 0], dtype=torch.int64, device="cuda")
    s["factor"] = torch.full((1,), 0.7, device="cuda")        # what clipping left
    return s


def _codes(x, positive=False):
    """Blocks of x as E4M3 codes and their scales."""
    x = x.view(-1, BLOCK)
    most = x.abs().amax(1)
    c = x * torch.where(most > 2.0 ** -100, 448.0 / most, 0.0)[:, None]
    if positive:
        c = torch.where(c > 0, c.clamp(min=2.0 ** -9), c)
    return c.to(E4).flatten(), most / 448.0


def _store(v, dtype):
    """v rounded to a storage format (FP8 casts saturate)."""
    most = MOST.get(dtype)
    return (v if most is None else v.clamp(-most, most)).to(dtype)


def _act(name, z):
    if name == "gelu":
        return z * 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    return z.clamp(min=0) if name == "relu" else torch.tanh(z) if name == "tanh" else torch.sigmoid(z)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _own(s, case, kind)
    if kind == "linear_bias":
        v = case["m"] ** -0.5 * (s["X"].float() @ s["W"].float()) + s["b"].float()
        out = {} if s["H"] is None else {"H": _store(v, s["H"].dtype)}
        if case["act"] != "none":
            v = FACTORS[case["act"]] * _act(case["act"], v)
        if s["skip"] is not None:
            v = HALF * s["skip"].float() + HALF * v
        return out | {"Y": _store(v, s["Y"].dtype)}
    if kind == "bias_grad":
        return [case["tokens"] ** -0.5 * G.float().sum(0) for G in s["G"]]
    if kind == "grad_norm":
        norm = s["g"].float().square().sum().sqrt()
        return {"norm": norm, "factor": (1.0 / norm).clamp(max=1.0)}
    g = s["g"].float() * s["factor"]
    b1, b2 = BETAS
    t = s["step"][:1] + 1
    fix1, fix2 = (1 - b1 ** t.double()).float(), (1 - b2 ** t.double()).float()
    small = case["states"] == "8bit"
    if small:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).flatten()
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).flatten().square()
    else:
        m, v = s["m"], s["v"]
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    root = v.sqrt()
    p, w = s["p"], _weights_end(case)
    p[:w] *= 1 - LR * DECAY                                   # (biases do not decay)
    p -= LR * (m / fix1) / (root / fix2.sqrt() + EPS)
    for c, part in zip(s["copies"], _parts(p, case)):
        c.copy_(_store(part, c.dtype))
    s["step"][:1] += 1
    if small:
        c, k = _codes(m)
        s["m"].copy_(c), s["m_scale"].copy_(k)
        c, k = _codes(root, True)
        s["v"].copy_(c), s["v_scale"].copy_(k)
    else:
        s["m"].copy_(m), s["v"].copy_(v)
    return _stepped(s)


def _stepped(s):
    return {k: s[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copies") if k in s} | {"step": s["step"][:1]}


def _own(s, case, kind):
    from paper_2303_11257_b200 import lib as L
    if kind == "linear_bias":
        act = {"none": L.US_ACT_NONE, "gelu": L.US_ACT_GELU, "relu": L.US_ACT_RELU, "tanh": L.US_ACT_TANH, "sigmoid": L.US_ACT_SIGMOID}[case["act"]]
        ep = None
        if act != L.US_ACT_NONE or s["skip"] is not None:
            ep = L.epilogue(act=act, act_out_scale=FACTORS.get(case["act"], 1.0), aux=s["H"], skip=s["skip"], skip_coef=HALF, out_coef=HALF)
        L.us_linear_fwd_bias(s["X"], s["W"], case["m"] ** -0.5, s["b"], s["Y"], s["scratch"], ep)
        return {"Y": s["Y"]} if s["H"] is None else {"H": s["H"], "Y": s["Y"]}
    if kind == "bias_grad":
        return L.us_bias_grad(s["G"], [case["tokens"] ** -0.5] * 2, s["db"])
    if kind == "grad_norm":
        if "plan" not in s:                                   # the list of tensors is laid out once, as a training loop does
            s["plan"] = L.mats(_parts(s["g"], case))
        L.us_grad_norm(s["plan"], 1.0, s["out"], s["scratch"])
        return {"norm": s["out"][0], "factor": s["out"][1]}
    if "plan" not in s:
        parts = {k: _parts(s[k], case) for k in ("p", "g", "m", "v")}
        scales = {}
        if case["states"] == "8bit":
            ends = [at // BLOCK for at in _places(case)[0]] + [_places(case)[1] // BLOCK]
            scales = {k: [s[k][i:j] for i, j in zip(ends, ends[1:])] for k in ("m_scale", "v_scale")}
        n = 2 * case["layers"]
        s["plan"] = L.adamw_tensors(parts["p"], parts["g"], parts["m"], parts["v"], **scales, copies=s["copies"] + [None] * (2 * n - len(s["copies"])),
                                    weight_decay=[DECAY] * n + [0.0] * n)
    L.us_adamw(s["plan"], s["step"], LR, BETAS, EPS, grad_factor=s["factor"])
    return _stepped(s)


def work(case):
    """Bytes of the inputs and results of a pass (each once), and the operations of its matrix products (else: of its elements)."""
    size = lambda name: TYPES[name].itemsize
    if case["kind"] == "linear_bias":
        T, m, n, e = case["tokens"], case["m"], case["n"], size(case["operand"])
        moved = e * (T * m + m * n) + T * n * (size(case["out"]) + (2 if case["kept"] else 0) + (size(case["skip"]) if case["skip"] != "none" else 0))
        return {"bytes": moved + n * size(case["bias"]), "flops": 2.0 * T * m * n}
    if case["kind"] == "bias_grad":
        n = case["tokens"] * (case["d"] + case["f"])
        return {"bytes": n * size(case["dtype"]) + 4 * (case["d"] + case["f"]), "flops": 1.0 * n}
    n = sum(math.prod(t) for t in _shapes(case))
    if case["kind"] == "grad_norm":
        return {"bytes": n * size(case["dtype"]) + 8, "flops": 2.0 * n}
    states = 16.0 if case["states"] == "f32" else 4 + 16 / BLOCK
    copied = 2 * case["layers"] * case["d"] * case["f"] * (size(case["copy"]) if case["copy"] != "none" else 0)
    return {"bytes": n * (8 + size(case["grad"]) + states) + copied, "flops": 15.0 * n}


# ---- the same results from the definitions in 64 bits.  The codes of states in 8 bits have no value here: rounding alone moves them by 2.6 % (2-norm).

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear_bias":
        z = torch.addmm(s["b"].double(), s["X"].double(), s["W"].double(), alpha=1 / math.sqrt(case["m"]))
        out = {"H": z.clone()} if case["kept"] else {}
        if case["act"] == "gelu":
            z = z * torch.special.ndtr(z)
        elif case["act"] == "relu":
            z = torch.where(z > 0, z, torch.zeros_like(z))
        elif case["act"] == "tanh":
            z = -torch.expm1(-2 * z) / (1 + torch.exp(-2 * z))
        elif case["act"] == "sigmoid":
            z = 1 / (1 + torch.exp(-z))
        z = z * FACTORS.get(case["act"], 1.0)
        if s["skip"] is not None:
            z = (s["skip"].double() + z) / math.sqrt(2)
        return out | {"Y": z}
    if kind == "bias_grad":
        one = torch.ones((1, case["tokens"]), dtype=torch.float64, device="cuda")
        return [(one @ G.double()).flatten() / math.sqrt(case["tokens"]) for G in s["G"]]
    if kind == "grad_norm":
        norm = torch.linalg.vector_norm(s["g"].double())
        return {"norm": norm, "factor": 1 / torch.clamp(norm, min=1.0)}
    t, (b1, b2) = case["steps"] + 1, BETAS
    g = s["g"].double() * s["factor"].double()
    small = case["states"] == "8bit"
    if small:
        m = s["m"].double() * s["m_scale"].double().repeat_interleave(BLOCK)
        root = s["v"].double() * s["v_scale"].double().repeat_interleave(BLOCK)
        v = root ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m = torch.lerp(g, m, b1)
    v = torch.lerp(g ** 2, v, b2)
    step = m * (LR / (1 - b1 ** t)) / ((v / (1 - b2 ** t)) ** 0.5 + EPS)
    kept = torch.ones_like(m)
    kept[:_weights_end(case)] -= LR * DECAY
    p = s["p"].double() * kept - step
    out = {"p": p, "copies": [part for _, part in zip(s["copies"], _parts(p, case))], "step": None}
    if small:
        return out | {"m": None, "v": None, "m_scale": m.abs().view(-1, BLOCK).amax(1) / 448, "v_scale": (v ** 0.5).view(-1, BLOCK).amax(1) / 448}
    return out | {"m": m, "v": v}
