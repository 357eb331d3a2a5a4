"""Operators of the layers that large language models have in the place of BERT's, as a list of measurable cases.

Kinds of work:
  gated_fwd  the hidden layer of a gated FFN block: both projections, the gate's activation and the product, with the
             copies of both projections that the backward pass reads, in 16 or in 8 bits (`us_ffn_gated_fwd`)
  gated_bwd  its backward pass down to both projections, from those copies: the second layer's input gradient and the
             gradients of gate and product (`us_ffn_gated_bwd`)
  qk_fwd     root-mean-square norms of the queries and of the keys, head by head, with the rotation of their positions
             (`us_qk_norm_fwd`)
  qk_bwd     its backward pass: gradients of queries, keys and both norm weights (`us_qk_norm_bwd`)

With h = alpha X Wg, u = alpha X Wu and z = s_in h (s_in = 1 here):
  A = alpha_g f(z) u;   dA = beta_x G W2^T,  dU = beta_u f(z) dA,  dH = beta_h f'(z) u dA  (h, u as the copies hold them)
and for each head x of D features, (c, s) the cosine and sine of the angle of its position and pair of features:
  n = w x / sqrt(mean(x^2) + eps),  y = (n_a c - n_b s, n_b c + n_a s) for each pair (a, b), other features y = n
  n' = the inverse rotation of dy,  dx = (w n' - xhat mean(w n' xhat)) / sqrt(mean(x^2) + eps),  dw = beta_w sum n' xhat

Activations and gradients are N(0, 1), the distribution unit scaling keeps them at.  `own` is false for the plain forms
below and true for the framework's kernels.
"""
import math

import torch

own = False

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": E4, "e5m2": E5}
OPERANDS = {"fp8": (E4, E5), "bf16": (torch.bfloat16, torch.bfloat16), "fp16": (torch.float16, torch.float16)}
MOST = {E4: 448.0, E5: 57344.0}
# 1 / rms f(Z) and 1 / rms f'(Z) for Z ~ N(0, 1): unit scale of the product and of both gradients
FACTORS = {"silu": (1.676532470331091, 1.6233202579524972), "gelu": (1.5335304411955353, 1.4811144127083482),
           "sigmoid": (1.8462285453386056, 4.722646085937974)}
EPS = 1e-6
SCRATCH = 4 << 20       # more than the workspace of any of the operators


def _gated(kind, tokens, d, f, operand, gate="silu", kept="bf16"):
    """kept: the type of the copies of both projections; none in evaluation."""
    return {"kind": kind, "tokens": tokens, "d": d, "f": f, "operand": operand, "gate": gate, "kept": kept}


def _qk(kind, tokens, heads, kv_heads, width, dtype, out, rotated=None, pairs="half", sequence=0):
    """sequence: tokens of a sequence, whose positions count from 0; 0: every token has a position of its own."""
    return {"kind": kind, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "width": width, "dtype": dtype, "out": out,
            "rotated": width if rotated is None else rotated, "pairs": pairs, "sequence": sequence}


def listed():
    cases = {
        # one token of one sequence being generated, BERT-large widths: latency counts
        "gated_fwd_token": _gated("gated_fwd", 1, 1024, 4096, "bf16", kept="none"),
        # a sub-batch left over at the end of an epoch in a block of pruned width: multiples of no tile
        "gated_fwd_ragged": _gated("gated_fwd", 1000, 528, 2096, "fp16", "gelu", "fp16"),
        # the FFN block of BERT-large on 16 x 512 tokens, gated, in training
        "gated_fwd_bert_large_bf16": _gated("gated_fwd", 8192, 1024, 4096, "bf16"),
        # a wider block on twice the tokens, FP8, with the copies for the backward pass in 8 bits: the largest
        "gated_fwd_wide_fp8": _gated("gated_fwd", 16384, 2048, 8192, "fp8", kept="e4m3"),
        # character language model (hidden 128, FFN 512, sequence 256): the smallest training step
        "gated_bwd_char_lm": _gated("gated_bwd", 256, 128, 512, "bf16"),
        # the backward passes of the BERT-large block, in 16 bits and in FP8 from copies of 8 bits
        "gated_bwd_bert_large_bf16": _gated("gated_bwd", 8192, 1024, 4096, "bf16"),
        "gated_bwd_bert_large_fp8": _gated("gated_bwd", 8192, 1024, 4096, "fp8", kept="e4m3"),
        # one token of one sequence being generated, four queries to a key
        "qk_fwd_token": _qk("qk_fwd", 1, 16, 4, 64, "bf16", "bf16"),
        # an attention layer of BERT-large on 16 x 512 tokens
        "qk_fwd_bert_large": _qk("qk_fwd", 8192, 16, 16, 64, "bf16", "bf16", sequence=512),
        # a long prompt of many documents in a packed batch, wide heads, FP8 attention operands
        "qk_fwd_wide": _qk("qk_fwd", 16384, 32, 8, 128, "bf16", "e4m3"),
        # half of an odd head width rotated, neighbouring features paired, a left-over sub-batch
        "qk_bwd_ragged": _qk("qk_bwd", 1000, 11, 11, 80, "fp16", "fp16", 40, "neighbours", 125),
        "qk_bwd_bert_large": _qk("qk_bwd", 8192, 16, 16, 64, "bf16", "bf16", sequence=512),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["gated_fwd", "gated_bwd", "qk_fwd", "qk_bwd"])
    while True:
        if kind.startswith("gated"):
            d = _log(rng, 128, 2048)
            operand = rng.choice(["fp8", "bf16", "fp16"])
            kept = rng.choice(["bf16" if operand == "fp8" else operand, "e4m3"] + (["none"] if kind == "gated_fwd" else []))
            c = _gated(kind, _log(rng, 1, 16384), d, _log(rng, 2 * d, min(8192, 4 * d)), operand, rng.choice(["silu", "silu", "gelu", "sigmoid"]), kept)
            if work(c)["flops"] <= 4.0 * 16384 * 2048 * 8192:
                return c
        else:
            width = rng.choice([32, 64, 64, 80, 96, 128, 128, 256, rng.randint(16, 256)])
            kv, tokens = rng.choice([1, 2, 4, 8, 11, 16]), _log(rng, 1, 16384)
            dtype = rng.choice(["bf16", "bf16", "fp16", "f32"])
            c = _qk(kind, tokens, kv * rng.choice([1, 1, 2, 4]), kv, width, dtype, rng.choice([dtype, "e4m3"] if kind == "qk_fwd" else [dtype]),
                    rng.choice([width // 2 * 2, width // 2 * 2, width // 4 * 2]), rng.choice(["half", "half", "neighbours"]),
                    rng.choice([0, _log(rng, 1, tokens)]))
            if work(c)["bytes"] <= 16384 * 40 * 128 * 6:
                return c


def _padded(rows, cols, dtype, parts=1):
    """`parts` matrices of rows x cols side by side in one, each on a boundary of 16 elements, as the library's alignment rule wants it."""
    pitch = (cols + 15) // 16 * 16
    m = torch.empty((rows, parts * pitch), dtype=dtype, device="cuda")
    return [m[:, i * pitch:i * pitch + cols] for i in range(parts)]


def _normal(gen, m):
    return m.copy_(torch.randn(m.shape, generator=gen, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)
    T, s = case["tokens"], {"case": case, "scratch": torch.zeros(SCRATCH, dtype=torch.uint8, device="cuda")}
    if case["kind"].startswith("gated"):
        d, f = case["d"], case["f"]
        act, grad = OPERANDS[case["operand"]]
        if case["kind"] == "gated_fwd":
            s["X"] = _normal(gen, _padded(T, d, act)[0])
            s["Wg"], s["Wu"] = (_normal(gen, m) for m in _padded(d, f, act, 2))
            s["A"] = _padded(T, f, act)[0]
            s["H"], s["U"] = _padded(T, f, TYPES[case["kept"]], 2) if case["kept"] != "none" else (None, None)
        else:
            s["G"], s["W2"] = _normal(gen, _padded(T, d, grad)[0]), _normal(gen, _padded(f, d, act)[0])
            s["H"], s["U"] = (_normal(gen, m) for m in _padded(T, f, TYPES[case["kept"]], 2))
            s["dH"], s["dU"] = _padded(T, f, grad, 2)
        return s
    D, dt, out = case["width"], TYPES[case["dtype"]], TYPES[case["out"]]
    at = [0, case["heads"] * D, (case["heads"] + case["kv_heads"]) * D]      # queries and keys are column slices of one matrix

    def both(dtype):
        m = torch.empty((T, at[2]), dtype=dtype, device="cuda")
        return [m[:, at[i]:at[i + 1]] for i in range(2)]
    s["x"] = [_normal(gen, m) for m in both(dt)]
    s["w"] = [(1 + 0.1 * torch.randn((D,), generator=gen, device="cuda")) for _ in range(2)]
    if case["kind"] == "qk_bwd":
        s["g"], s["dw"] = [_normal(gen, m) for m in both(dt)], [torch.empty((D,), device="cuda") for _ in range(2)]
    s["y"] = both(out)
    # (cos, sin) of position times 10000^(-2 i / rotated), made in 64 bits and kept in 32
    P = case["sequence"] or 32768
    i = torch.arange(case["rotated"] // 2, device="cuda", dtype=torch.float64)
    angle = torch.arange(P, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-2 * i / max(1, case["rotated"]))
    s["table"] = torch.stack([angle.cos(), angle.sin()], -1).flatten(1).float()
    s["positions"] = None if case["sequence"] else torch.randint(0, P, (T,), generator=gen, device="cuda", dtype=torch.int32)
    return s


def _store(v, dtype):
    """v rounded to a storage format (FP8 casts saturate)."""
    most = MOST.get(dtype)
    return (v if most is None else v.clamp(-most, most)).to(dtype)


def _gate(name, z):
    """f and f' of the gate."""
    if name == "gelu":
        phi = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = torch.sigmoid(z)
    return (z * s, s * (1 + z * (1 - s))) if name == "silu" else (s, s * (1 - s))


def _angles(s):
    """cos and sin of every token and pair: [tokens, 1, pairs]."""
    t = s["table"].view(s["table"].shape[0], -1, 2)
    T = s["case"]["tokens"]
    at = s["positions"].long() if s["positions"] is not None else torch.arange(T, device="cuda") % s["case"]["sequence"]
    t = t[at][:, None]
    return t[..., 0], t[..., 1]


def _rotated(v, c, s, case, back=False):
    """v [tokens, heads, width] with the pairs of its rotated features turned by their angles, or back."""
    r, half = case["rotated"], case["pairs"] == "half"
    a, b = (v[..., :r // 2], v[..., r // 2:r]) if half else (v[..., :r:2], v[..., 1:r:2])
    if back:
        s = -s
    a, b = a * c - b * s, b * c + a * s
    return torch.cat([torch.cat([a, b], -1) if half else torch.stack([a, b], -1).flatten(-2), v[..., r:]], -1)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _own(s, case, kind)
    if kind == "gated_fwd":
        X, alpha = s["X"].float(), case["d"] ** -0.5
        h, u = alpha * (X @ s["Wg"].float()), alpha * (X @ s["Wu"].float())
        A = _store(FACTORS[case["gate"]][0] * _gate(case["gate"], h)[0] * u, s["A"].dtype)
        return {"A": A} if s["H"] is None else {"A": A, "H": _store(h, s["H"].dtype), "U": _store(u, s["H"].dtype)}
    if kind == "gated_bwd":
        dA = case["d"] ** -0.5 * (s["G"].float() @ s["W2"].float().T)
        f, df = _gate(case["gate"], s["H"].float())
        beta_u, beta_h = FACTORS[case["gate"]]
        return {"dH": _store(beta_h * df * s["U"].float() * dA, s["dH"].dtype), "dU": _store(beta_u * f * dA, s["dU"].dtype)}
    T, D = case["tokens"], case["width"]
    c, sn = _angles(s)
    out = {}
    for name, k in (("q", 0), ("k", 1)):
        x, w = s["x"][k].float().reshape(T, -1, D), s["w"][k]
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        if kind == "qk_fwd":
            out[name] = _store(_rotated(x * r * w, c, sn, case), s["y"][k].dtype).flatten(1)
            continue
        n, xhat = _rotated(s["g"][k].float().reshape(T, -1, D), c, sn, case, back=True), x * r
        out["d" + name] = _store(r * (n * w - xhat * (n * w * xhat).mean(-1, keepdim=True)), s["y"][k].dtype).flatten(1)
        out["dw_" + name] = (T * x.shape[1]) ** -0.5 * (n * xhat).sum((0, 1))
    return out


def _own(s, case, kind):
    from paper_2303_11257_b200 import lib as L
    if kind == "gated_fwd":
        L.us_ffn_gated_fwd(case["gate"], s["X"], s["Wg"], s["Wu"], case["d"] ** -0.5, s["A"], s["scratch"], H=s["H"], U=s["U"],
                           act_out_scale=FACTORS[case["gate"]][0])
        return {"A": s["A"]} if s["H"] is None else {"A": s["A"], "H": s["H"], "U": s["U"]}
    if kind == "gated_bwd":
        beta_u, beta_h = FACTORS[case["gate"]]
        L.us_ffn_gated_bwd(case["gate"], s["G"], s["W2"], case["d"] ** -0.5, s["H"], s["U"], s["dH"], s["dU"], s["scratch"], beta_h=beta_h, beta_u=beta_u)
        return {"dH": s["dH"], "dU": s["dU"]}
    place = dict(table=s["table"], positions=s["positions"], period=case["sequence"], neighbours=case["pairs"] == "neighbours")
    if kind == "qk_fwd":
        L.us_qk_norm_fwd(s["x"], s["w"], s["y"], case["width"], EPS, **place)
        return {"q": s["y"][0], "k": s["y"][1]}
    T = case["tokens"]
    L.us_qk_norm_bwd(s["x"], s["w"], s["g"], s["y"], s["dw"], case["width"], EPS, s["scratch"],
                     beta_w=[(T * case["heads"]) ** -0.5, (T * case["kv_heads"]) ** -0.5], **place)
    return {"dq": s["y"][0], "dk": s["y"][1], "dw_q": s["dw"][0], "dw_k": s["dw"][1]}


def work(case):
    """Bytes of the inputs and results of a pass (each once), and the operations of its matrix products (of a norm: of its elements)."""
    T = case["tokens"]
    if case["kind"].startswith("gated"):
        d, f, e = case["d"], case["f"], 1 if case["operand"] == "fp8" else 2
        kept = 2 * T * f * {"none": 0, "e4m3": 1}.get(case["kept"], 2)
        if case["kind"] == "gated_fwd":
            return {"bytes": e * (T * d + 2 * d * f + T * f) + kept, "flops": 4.0 * T * d * f}
        return {"bytes": e * (T * d + d * f + 2 * T * f) + kept, "flops": 2.0 * T * d * f}
    n = T * (case["heads"] + case["kv_heads"]) * case["width"]
    e, o = TYPES[case["dtype"]].itemsize, TYPES[case["out"]].itemsize
    table = 4 * case["rotated"] * min(T, case["sequence"] or 32768) + (4 * T if not case["sequence"] else 0) + 8 * case["width"]
    if case["kind"] == "qk_fwd":
        return {"bytes": n * (e + o) + table, "flops": 10.0 * n}
    return {"bytes": n * (2 * e + o) + table + 8 * case["width"], "flops": 20.0 * n}


# ---- the same results from the definitions in 64 bits, written with complex numbers and closed forms of their own.  Gradients that are
# rounded to E5M2 have no value here: that rounding alone moves them by 5.3 % (2-norm), more than a computation may be off.

def _gate64(name, z):
    if name == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * (2 * math.pi) ** -0.5 * torch.exp(z.square() / -2)
    m, p = 1 / (1 + torch.exp(z)), 1 / (1 + torch.exp(-z))
    return (p * z, p + z * p * m) if name == "silu" else (p, p * m)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "gated_fwd":
        X, k = s["X"].double(), 1 / math.sqrt(case["d"])
        h = torch.mm(X, s["Wg"].double()).mul_(k)
        u = torch.mm(X, s["Wu"].double()).mul_(k)
        A = _gate64(case["gate"], h)[0].mul_(u).mul_(FACTORS[case["gate"]][0])
        return {"A": A} if s["H"] is None else {"A": A, "H": h, "U": u}
    if kind == "gated_bwd":
        if s["dH"].dtype == E5:
            return None
        dA = torch.mm(s["G"].double(), s["W2"].double().T) / math.sqrt(case["d"])
        f, df = _gate64(case["gate"], s["H"].double())
        return {"dH": df.mul_(s["U"].double()).mul_(dA).mul_(FACTORS[case["gate"]][1]), "dU": f.mul_(dA).mul_(FACTORS[case["gate"]][0])}
    T, D, r = case["tokens"], case["width"], case["rotated"]
    t = torch.view_as_complex(s["table"].double().view(s["table"].shape[0], r // 2, 2))
    place = s["positions"] if s["positions"] is not None else torch.remainder(torch.arange(T, device="cuda"), case["sequence"])
    turn = t.index_select(0, place.long()).unsqueeze(1)

    def times(v, z):                                     # the pairs of v as complex numbers, times z
        a, rest = v[..., :r], v[..., r:]
        if case["pairs"] == "half":
            p = torch.complex(*a.unflatten(-1, (2, r // 2)).unbind(-2)) * z
            return torch.cat([p.real, p.imag, rest], -1)
        p = torch.view_as_complex(a.unflatten(-1, (r // 2, 2)).contiguous()) * z
        return torch.cat([torch.view_as_real(p).flatten(-2), rest], -1)

    out = {}
    for k, name in enumerate("qk"):
        x, w = s["x"][k].double().unflatten(-1, (-1, D)), s["w"][k].double()
        size = (torch.linalg.vector_norm(x, dim=-1, keepdim=True).square() / D + EPS).sqrt()
        if kind == "qk_fwd":
            out[name] = times(x / size * w, turn).flatten(1)
        else:
            n = times(s["g"][k].double().unflatten(-1, (-1, D)), turn.conj())
            v = n * w
            out["d" + name] = (v / size - x * (v * x).sum(-1, keepdim=True) / (D * size ** 3)).flatten(1)
            out["dw_" + name] = torch.einsum("thd,thd->d", n, x / size) / math.sqrt(T * x.shape[1])
    return out
