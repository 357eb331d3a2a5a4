"""us_bias_grad against the oracle.

Tolerance in units of u = 2^-24: a thread adds every 32nd (rows that do not start on 16-byte boundaries: every 8th) row of its part, then 2 + 8 + 8 sums
join, and the factor is one product more: (rows of a thread + 20) of beta * the sum of magnitudes; 16-bit results half a step more."""
import numpy as np
import pytest
import torch

from oracle import ops as O
from tests import util as U

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


def _lib():
    from paper_2303_11257_b200 import lib
    return lib


def _part(rows, cols, fmt, ld, out, seed, shift=0):
    """A matrix among NaNs, its gradient, and the check of it."""
    dt = U.TORCH_OF[fmt]
    x = np.random.default_rng(seed).standard_normal((rows, cols))
    size = max(0, (rows - 1) * ld + cols)
    buf = torch.full((size + shift + 1,), float("nan")).to(dt).cuda()
    G = torch.as_strided(buf, (rows, cols), (ld, 1), shift) if rows else buf[:0].view(0, cols) if not cols else torch.empty((0, cols), dtype=dt, device="cuda")
    if rows:
        G.copy_(torch.from_numpy(np.float32(x)).cuda().to(dt))
    whole = torch.full((cols + 2,), -7.0, dtype=U.TORCH_OF[out], device="cuda")

    def check(beta):
        g = U.host_values(G) if rows else np.zeros((0, cols))
        want = O.bias_grad(g, beta)
        tol = (rows / 8 + 20) * u * abs(beta) * np.abs(g).sum(0)
        if out != "f32":
            tol = tol + 0.5 * U.ulp_of(np.abs(want) + tol, out)
        got = U.host_values(whole)
        assert (np.abs(got[1:-1] - want) <= tol).all(), (rows, cols, fmt, ld, float((np.abs(got[1:-1] - want) - tol).max()))
        assert got[0] == got[-1] == -7.0
    return G, whole[1:-1], check


FORMATS = ["f32", "bf16", "fp16", "e4m3", "e5m2"]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 4096, 0), (31, 128, 0), (32, 129, 0), (33, 80, 16), (64, 100, 12), (65, 1000, 0), (129, 48, 0), (257, 520, 8), (1000, 2096, 0),
                                           (4097, 300, 4), (1025, 33, 15), (0, 50, 0)])
def test_shapes(rows, cols, pad, fmt):
    G, db, check = _part(rows, cols, fmt, cols + pad, "f32", rows + cols)
    _lib().us_bias_grad([G], [0.37], [db])
    check(0.37)


@pytest.mark.parametrize("fmt", FORMATS)
def test_the_last_row_is_not_read_past_its_end(fmt):
    """Rows on 16-byte boundaries whose last column is not at one: nothing lies behind the last row."""
    es = U.TORCH_OF[fmt].itemsize
    cols = 16 // es * 9 + 1
    for rows in (1, 2, 200, 300):
        G, db, check = _part(rows, cols, fmt, 16 // es * 10, "f32", rows)
        _lib().us_bias_grad([G], None, [db])
        check(1.0)


def test_eight_matrices_of_all_kinds_at_once():
    parts = [_part(r, c, f, c + p, o, r + c, s) for r, c, f, p, o, s in
             [(8192, 1024, "e5m2", 0, "f32", 0), (300, 70, "bf16", 2, "bf16", 0), (1, 5000, "f32", 0, "fp16", 0), (0, 9, "f32", 0, "f32", 0), (77, 333, "fp16", 1, "f32", 1),
              (2000, 16, "e4m3", 0, "f32", 3), (5, 1, "f32", 7, "bf16", 2), (3000, 700, "bf16", 4, "fp16", 0)]]
    beta = [0.01, -1.0, 2.0, 3.0, 0.5, 0.1, 1.0, 0.02]
    db = _lib().us_bias_grad([p[0] for p in parts], beta, [p[1] for p in parts])
    first = [d.clone() for d in db]
    for p, b in zip(parts, beta):
        p[2](b)
    for _ in range(3):
        _lib().us_bias_grad([p[0] for p in parts], beta, db)
        assert all(torch.equal(x, y) for x, y in zip(first, db))


def test_rows_beyond_32_bits():
    """Elements past 2^32: a row pitch of 2^31 / 600 and 1400 rows, of which few columns are read."""
    rows, ld, cols = 1400, 3600000, 20
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    buf = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    G = torch.as_strided(buf, (rows, cols), (ld, 1))
    G.copy_(torch.randn(rows, cols, device="cuda"))
    db = torch.empty(cols, device="cuda")
    _lib().us_bias_grad([G], [0.5], [db])
    want = O.bias_grad(U.host_values(G), 0.5)
    assert (np.abs(U.host_values(db) - want) <= 200 * u * 0.5 * np.abs(U.host_values(G)).sum(0)).all()


def test_nan_and_infinity_stay_in_their_columns():
    G = torch.ones((500, 300), device="cuda").to(torch.bfloat16)
    G[3, 7], G[400, 299] = float("nan"), float("inf")
    db = torch.empty(300, device="cuda")
    _lib().us_bias_grad([G], None, [db])
    assert torch.isnan(db[7]) and torch.isinf(db[299]) and int((db == 500).sum()) == 298


def test_captured_and_on_another_stream():
    G = torch.randn((3000, 500), device="cuda")
    db, other = torch.empty(500, device="cuda"), torch.empty(500, device="cuda")
    _lib().us_bias_grad([G], None, [db])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _lib().us_bias_grad([G], None, [other])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(db, other)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _lib().us_bias_grad([G], None, [other])
    G.mul_(2)
    g.replay()
    assert torch.equal(other, 2 * db)
