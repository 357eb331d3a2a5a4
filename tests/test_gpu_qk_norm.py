"""us_qk_norm_fwd / us_qk_norm_bwd / us_rotary_table against the oracle.

Tolerances, in units of 2^-24 (half a float32 step): a lane adds 16 squares and a group 5 times, all positive, so mean(x^2) is off by at most
22 units and its root by 11; rsqrtf by 2 steps, 4 units; with the products and the rotation's two, n by 20.  A turned feature
is off by that much of |n_a| + |n_b|: 1.2e-6, taken as 1.5e-6.  The gradient's second term holds 1 / size three times and a second
sum: 3 * 15 + 22 + 8 = 75 units, 4.5e-6, taken as 5e-6 of r (|g_a| + |g_b|) |w| + |xhat| mean |u xhat|.  A weight gradient adds at most 2 terms in
a lane of each of four steps, then 5 times over groups, 8 over warps, 10 + 5 over CTAs, all rounded relative to the sum of magnitudes: 36 + 15 + 3 units of
it, 3.3e-6, taken as 4e-6.  What is stored in fewer bits adds half a step of its format."""
import numpy as np
import pytest
import torch

from oracle import formats as F
from oracle import ops as O
from tests import util as U

pytestmark = pytest.mark.gpu


def _lib():
    from paper_2303_11257_b200 import lib
    return lib


def _pad(k, fmt):
    es = {"f32": 4, "bf16": 2, "fp16": 2}.get(fmt, 1)
    return (k * es + 15) // 16 * 16 // es


def _magnitude(v, r, neighbours):
    """|v_a| + |v_b| at both features of a pair, |v| elsewhere."""
    m = np.abs(v)
    out = m.copy()
    ia = np.arange(0, r, 2) if neighbours else np.arange(r // 2)
    ib = ia + 1 if neighbours else ia + r // 2
    out[..., ia] = out[..., ib] = m[..., ia] + m[..., ib]
    return out


def _step(ref, fmt):
    return 0.0 if fmt == "f32" else 0.5 * U.ulp_of(ref, fmt) * (1 + 1e-6)


def _check(got, ref, tol, fmt, what):
    g = U.host_values(got)
    ref = np.asarray(ref)
    if fmt in ("e4m3", "e5m2"):
        ref = np.clip(ref, -F.FORMATS[fmt].max_finite, F.FORMATS[fmt].max_finite)
    bad = ~(np.abs(g - ref) <= tol + _step(np.abs(ref) + tol, fmt))
    assert not bad.any(), (what, int(bad.sum()), float(np.abs(g - ref)[bad].max()))


def _case(rows, heads, width, rotated, neighbours, dt, out, offset, where, bwd, w_fmt="f32", seed=0):
    """One call for queries and keys against the oracle; offset: columns before the first head, so that slices start anywhere."""
    L = _lib()
    rng = np.random.default_rng(seed + rows + 7 * width)
    table_h = np.float32(O.rotary_table(64, rotated)) if rotated else None
    table = None if table_h is None else torch.from_numpy(table_h).cuda()
    if where == "given":
        at = rng.integers(0, 64, rows)
        place = dict(positions=torch.from_numpy(at.astype(np.int32)).cuda())
    elif where == "period":
        at = 3 + np.arange(rows) % 13
        place = dict(start=3, period=13)
    else:
        at = np.arange(rows)
        place = {}
    cols = sum(heads) * width
    whole = rng.standard_normal((rows, offset + cols)).astype(np.float32)
    wholeg = rng.standard_normal((rows, offset + cols)).astype(np.float32)
    buf = U.to_device(whole, dt, ld=_pad(offset + cols, dt) + 16)
    bufg = U.to_device(wholeg, dt, ld=_pad(offset + cols, dt) + 16)
    outb = U.empty(rows, offset + cols, out, ld=_pad(offset + cols, out) + 16)
    full = torch.as_strided(outb.view(torch.uint8) if outb.element_size() == 1 else outb, (rows, outb.stride(0)), (outb.stride(0), 1)) if rows else outb
    X, G, Y, Xv, Gv, Ws, Wv, c = [], [], [], [], [], [], [], offset
    for k, h in enumerate(heads):
        sl = slice(c, c + h * width)
        X.append(buf[:, sl]); G.append(bufg[:, sl]); Y.append(outb[:, sl])
        Xv.append(U.values_of(whole, dt)[:, sl]); Gv.append(U.values_of(wholeg, dt)[:, sl])
        w = (1 + 0.3 * rng.standard_normal((1, width))).astype(np.float32)
        Ws.append(U.to_device(w, w_fmt)[0]); Wv.append(U.values_of(w, w_fmt)[0])
        c += h * width
    eps = 1e-5
    if not bwd:
        L.us_qk_norm_fwd(X, Ws, Y, width, eps, table=table, neighbours=neighbours, **place)
        for k in range(len(heads)):
            ref = O.qk_norm_fwd(Xv[k], Wv[k], width, eps, table_h, at, neighbours)
            n = O.qk_norm_fwd(Xv[k], Wv[k], width, eps).reshape(rows, heads[k], width)
            _check(Y[k], ref, 1.5e-6 * _magnitude(n, rotated, neighbours).reshape(rows, heads[k] * width), out, (k, rows, width))
    else:
        ws = torch.empty(L.us_qk_norm_bwd_workspace_bytes(width), dtype=torch.uint8, device="cuda")
        beta_w = [0.5, 0.25, 0.125][: len(heads)]
        dw = [torch.full((width,), 9.0, device="cuda") for _ in heads]
        L.us_qk_norm_bwd(X, Ws, G, Y, dw, width, eps, ws, beta_x=0.75, beta_w=beta_w, table=table, neighbours=neighbours, **place)
        for k in range(len(heads)):
            dX, dwr = O.qk_norm_bwd(Xv[k], Wv[k], Gv[k], width, eps, 0.75, beta_w[k], table_h, at, neighbours)
            x, g = (v.reshape(rows, heads[k], width) for v in (Xv[k], Gv[k]))
            size = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
            m = _magnitude(g, rotated, neighbours)
            tol = 0.75 / size * (m * np.abs(Wv[k]) + np.abs(x / size) * (m * np.abs(Wv[k]) * np.abs(x / size)).mean(-1, keepdims=True))
            _check(Y[k], dX, 5e-6 * tol.reshape(rows, heads[k] * width), out, (k, rows, width))
            lim = 4e-6 * beta_w[k] * (m * np.abs(x / size)).sum((0, 1))
            err = np.abs(dw[k].double().cpu().numpy() - dwr)
            assert (err <= lim).all(), (k, float((err / np.maximum(lim, 1e-30)).max()))
    if rows:
        rest = torch.cat([full[:, :offset], full[:, offset + cols:]], 1).float()
        assert not rest.any()                                    # nothing outside the matrices is written


VEC = [(1, (4, 1), 64, 64, False), (5, (1,), 8, 0, False), (37, (16, 4), 64, 64, False), (130, (3, 3), 128, 128, True), (64, (8, 2, 2), 96, 64, False),
       (33, (5, 1), 256, 256, False), (21, (2, 1), 512, 512, True), (50, (11, 11), 80, 40, True), (40, (6, 2), 72, 48, False), (3000, (12, 12), 64, 32, False),
       (2, (33, 1), 16, 16, True), (9, (7, 7), 24, 8, True), (600, (40, 8), 128, 128, False)]
ODD = [(1, (1,), 1, 0, False), (7, (3, 2), 73, 72, False), (19, (2, 2), 33, 10, True), (5, (2,), 1024, 1024, False), (4, (1, 1), 999, 2, True),
       (260, (9, 3), 66, 66, False), (31, (4, 4), 40, 24, False)]


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("where", ["given", "period"])
@pytest.mark.parametrize("shape", VEC + ODD)
@pytest.mark.parametrize("dt", ["bf16", "fp16", "f32"])
def test_matches_the_oracle(shape, dt, where, bwd):
    rows, heads, width, rotated, neighbours = shape
    _case(rows, heads, width, rotated, neighbours, dt, dt, 0, where, bwd)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("out", ["f32", "bf16", "fp16", "e4m3", "e5m2"])
@pytest.mark.parametrize("offset", [0, 8, 1])
def test_output_types_and_slices_that_start_anywhere(out, offset, bwd):
    _case(45, (6, 2), 64, 64, False, "bf16", out, offset, "given", bwd)
    _case(45, (6, 2), 80, 32, True, "f32", out, offset, "rows", bwd, w_fmt="bf16")


@pytest.mark.parametrize("bwd", [False, True])
def test_no_rows_no_heads(bwd):
    _case(0, (4, 2), 64, 64, False, "bf16", "bf16", 0, "rows", bwd)
    L = _lib()
    none = torch.empty((3, 0), dtype=torch.bfloat16, device="cuda")
    L.us_qk_norm_fwd([none], None, [none], 64, 1e-6)
    torch.cuda.synchronize()


def test_positions_outside_the_table_are_nan_and_others_are_not():
    L = _lib()
    for width in (64, 63):
        X = torch.randn(6, 2 * width, device="cuda")
        Y = torch.empty_like(X)
        at = torch.tensor([0, -1, 31, 32, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
        L.us_qk_norm_fwd([X], None, [Y], width, 0.0, table=L.rotary_table(32, 16), positions=at)
        y = Y.view(6, 2, width)
        assert torch.isnan(y[[1, 3, 4, 5], :, :16]).all() and torch.isfinite(y[[0, 2]]).all() and torch.isfinite(y[:, :, 16:]).all()


@pytest.mark.parametrize("width", [64, 63])
def test_values_that_are_not_finite_stay_in_their_head(width):
    L = _lib()
    X = torch.randn(5, 3 * width, device="cuda").to(torch.bfloat16)
    G, w = torch.randn_like(X), torch.ones(width, device="cuda")
    clean = [torch.empty_like(X) for _ in range(2)]
    ws, dw = torch.empty(L.us_qk_norm_bwd_workspace_bytes(width), dtype=torch.uint8, device="cuda"), torch.empty(width, device="cuda")
    table = L.rotary_table(8, 32)

    def both(x, out):
        L.us_qk_norm_fwd([x], [w], [out[0]], width, 0.0, table=table)
        L.us_qk_norm_bwd([x], [w], [G], [out[1]], [dw], width, 0.0, ws, table=table)
    both(X, clean)
    bad, out = X.clone(), [torch.empty_like(X) for _ in range(2)]
    bad[1, width + 3], bad[2, 5], bad[4, :width] = float("nan"), float("inf"), 0.0            # (a head of zeros without eps: 0 / 0)
    both(bad, out)
    hit = torch.zeros(5, 3, dtype=torch.bool, device="cuda")
    hit[1, 1] = hit[2, 0] = hit[4, 0] = True
    for o, c in zip(out, clean):
        o, c = o.view(5, 3, width), c.view(5, 3, width)
        assert torch.equal(o[~hit], c[~hit]) and torch.isnan(o[1, 1]).all() and torch.isnan(o[4, 0]).all() and torch.isnan(o[2, 0]).any()


def test_in_place_and_repeated_calls_give_the_same_bits():
    L = _lib()
    for width, heads in ((64, 16), (50, 3)):
        X = torch.randn(700, heads * width, device="cuda").to(torch.bfloat16)
        G, w, table = torch.randn_like(X), 1 + 0.1 * torch.randn(width, device="cuda"), L.rotary_table(700, width // 2 * 2)
        ws = torch.empty(L.us_qk_norm_bwd_workspace_bytes(width), dtype=torch.uint8, device="cuda")
        Y, dX, dw = torch.empty_like(X), torch.empty_like(X), torch.empty(width, device="cuda")
        L.us_qk_norm_fwd([X], [w], [Y], width, 1e-6, table=table)
        L.us_qk_norm_bwd([X], [w], [G], [dX], [dw], width, 1e-6, ws, table=table)
        x, g, g2, dw2 = X.clone(), G.clone(), G.clone(), torch.empty_like(dw)
        L.us_qk_norm_fwd([x], [w], [x], width, 1e-6, table=table)
        L.us_qk_norm_bwd([X], [w], [g], [g], [dw2], width, 1e-6, ws, table=table)
        assert torch.equal(x, Y) and torch.equal(g, dX) and torch.equal(dw, dw2)
        x = X.clone()
        L.us_qk_norm_bwd([x], [w], [g2], [x], [dw2], width, 1e-6, ws, table=table)
        assert torch.equal(x, dX) and torch.equal(dw, dw2)


def test_captured_and_replayed_on_another_stream():
    L = _lib()
    width, rows = 64, 300
    X, G = (torch.randn(rows, 8 * width, device="cuda").to(torch.bfloat16) for _ in range(2))
    w, table = torch.ones(width, device="cuda"), L.rotary_table(4096, width)
    at = torch.arange(rows, device="cuda", dtype=torch.int32)
    ws = torch.empty(L.us_qk_norm_bwd_workspace_bytes(width), dtype=torch.uint8, device="cuda")
    Y, dX, dw = torch.empty_like(X), torch.empty_like(X), torch.empty(width, device="cuda")

    def step():
        L.us_qk_norm_fwd([X], [w], [Y], width, 1e-6, table=table, positions=at)
        L.us_qk_norm_bwd([X], [w], [G], [dX], [dw], width, 1e-6, ws, table=table, positions=at)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    X.copy_(torch.randn_like(X)); at.add_(1000)
    g.replay()
    got = [t.clone() for t in (Y, dX, dw)]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for t in (Y, dX, dw):
        t.zero_()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        step()
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (Y, dX, dw)))


@pytest.mark.parametrize("x_fmt,g_fmt", [("bf16", "bf16"), ("f32", "bf16"), ("fp16", "f32")])
@pytest.mark.parametrize("place", [dict(start=17), dict(start=5, period=1), dict(period=200), dict(period=41, start=2)])
def test_matrices_of_their_own_pitches_and_types(x_fmt, g_fmt, place):
    """Queries of one type and keys of another, gradients with other pitches and types, every way to say where rows are."""
    L = _lib()
    rng = np.random.default_rng(11)
    rows, width, heads, eps = 83, 64, (5, 2), 1e-5
    table_h = np.float32(O.rotary_table(120, width))
    table = torch.from_numpy(table_h).cuda()
    at = place.get("start", 0) + (np.arange(rows) % place["period"] if place.get("period") else np.arange(rows))
    x_fmts = (x_fmt, "bf16")
    Xh, Gh = ([rng.standard_normal((rows, h * width)).astype(np.float32) for h in heads] for _ in range(2))
    X = [U.to_device(x, f, ld=x.shape[1] + 8 * (k + 1)) for k, (x, f) in enumerate(zip(Xh, x_fmts))]
    G = [U.to_device(g, g_fmt, ld=g.shape[1] + 24) for g in Gh]
    w = [torch.ones(width, device="cuda") * (1 + k) for k in range(2)]
    Y, dX, dw = [torch.empty_like(x, dtype=torch.float32) for x in _f32_like(X)], [torch.empty_like(x, dtype=torch.float32) for x in _f32_like(X)], [torch.empty(width, device="cuda") for _ in range(2)]
    ws = torch.empty(L.us_qk_norm_bwd_workspace_bytes(width), dtype=torch.uint8, device="cuda")
    L.us_qk_norm_fwd(X, w, Y, width, eps, table=table, **place)
    L.us_qk_norm_bwd(X, w, G, dX, dw, width, eps, ws, table=table, **place)
    for k in range(2):
        x, g = U.values_of(Xh[k], x_fmts[k]), U.values_of(Gh[k], g_fmt)
        n = O.qk_norm_fwd(x, [1.0 + k] * width, width, eps).reshape(rows, heads[k], width)
        _check(Y[k], O.qk_norm_fwd(x, [1.0 + k] * width, width, eps, table_h, at), 1.5e-6 * _magnitude(n, width, False).reshape(rows, -1), "f32", "Y")
        ref, dwr = O.qk_norm_bwd(x, [1.0 + k] * width, g, width, eps, 1.0, 1.0, table_h, at)
        xv, m = x.reshape(rows, heads[k], width), _magnitude(g.reshape(rows, heads[k], width), width, False) * (1.0 + k)
        size = np.sqrt((xv * xv).mean(-1, keepdims=True) + eps)
        _check(dX[k], ref, (5e-6 / size * (m + np.abs(xv / size) * (m * np.abs(xv / size)).mean(-1, keepdims=True))).reshape(rows, -1), "f32", "dX")
        assert (np.abs(dw[k].double().cpu().numpy() - dwr) <= 4e-6 * (m / (1.0 + k) * np.abs(xv / size)).sum((0, 1))).all()


def _f32_like(X):
    return [torch.empty(x.shape, device="cuda") for x in X]


def test_many_rows_and_offsets_beyond_32_bits():
    """Rows 1.6 million elements apart: the last one starts 4.6e9 elements into its buffer."""
    L = _lib()
    rows, pitch, width = 2900, 1_600_000, 64
    buf = torch.empty(rows * pitch, dtype=torch.bfloat16, device="cuda")
    X = torch.as_strided(buf, (rows, 2 * width), (pitch, 1))
    x = torch.randn(rows, 2 * width, device="cuda").to(torch.bfloat16)
    X.copy_(x)
    table = L.rotary_table(rows, width)
    Y, want = torch.as_strided(buf, (rows, 2 * width), (pitch, 1), 128), torch.empty_like(x)
    L.us_qk_norm_fwd([x], None, [want], width, 1e-6, table=table)
    L.us_qk_norm_fwd([X], None, [Y], width, 1e-6, table=table)
    assert torch.equal(Y, want)
    del buf, X, Y


def test_table():
    """float32 values of angles that are formed in 64 bits: half a step of the cosine, and what 1e-15 of the angle moves it by."""
    L = _lib()
    for rows, rotated, base, scale, first in ((100, 64, 10000.0, 1.0, 0), (50, 6, 500000.0, 0.25, 1 << 20), (3, 2, 10.0, 1.0, 0), (4, 0, 10.0, 1.0, 0)):
        t = torch.empty((rows, rotated + 4), device="cuda")[:, :rotated]
        L.us_rotary_table(t, base, scale, first)
        ref = O.rotary_table(rows, rotated, base, scale, first)
        assert np.all(np.abs(t.double().cpu().numpy() - ref) <= 2.0 ** -25 + 2e-9)


def test_table_rows_more_than_32_bits_apart():
    """A table whose rows lie 2^32 and more elements apart turns as the same table in one piece does."""
    L = _lib()
    rows, width = 5, 64
    X = torch.randn(rows, 4 * width, device="cuda").to(torch.bfloat16)
    at = torch.tensor([1, 0, 1, 1, 0], dtype=torch.int32, device="cuda")
    near = L.rotary_table(64, width)[[7, 40]]
    ws, w = torch.empty(L.us_qk_norm_bwd_workspace_bytes(width), dtype=torch.uint8, device="cuda"), torch.ones(width, device="cuda")

    def both(table):
        Y, dX, dw = torch.empty_like(X), torch.empty_like(X), torch.empty(width, device="cuda")
        L.us_qk_norm_fwd([X], [w], [Y], width, 1e-6, table=table, positions=at)
        L.us_qk_norm_bwd([X], [w], [X], [dX], [dw], width, 1e-6, ws, table=table, positions=at)
        return Y, dX, dw
    want = both(near)
    for pitch in (2 ** 32, 2 ** 32 + 64):
        buf = torch.zeros(pitch + width, device="cuda")
        far = torch.as_strided(buf, (2, width), (pitch, 1))
        far.copy_(near)
        assert all(torch.equal(a, b) for a, b in zip(both(far), want)), pitch
        del buf, far
