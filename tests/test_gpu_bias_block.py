"""An FFN block with biases and the optimiser that updates it: runs of the operators together, against the oracle's chain.  Each operator is checked strictly
on its own; here tensors early in the chain are held to a step of their format and later ones statistically, as for the other blocks."""
import numpy as np
import pytest
import torch

from oracle import ops as O
from tests import util as U
from tests.test_gpu_gated_block import _host, _near
from tests.test_gpu_launch_counts import _kernels

pytestmark = pytest.mark.gpu


def _make(T, d, f, seed=61):
    X, W1, W2, G = _host(seed, (T, d), (d, f), (f, d), (T, d))
    rng = np.random.default_rng(seed)
    return (X, W1, W2, G), rng.standard_normal(f).astype(np.float32), rng.standard_normal(d).astype(np.float32)


@pytest.mark.parametrize("T,d,f", [(96, 64, 80), (300, 144, 400), (1024, 272, 1104), (1, 128, 512)])
@pytest.mark.parametrize("operand", ["fp8", "bf16", "fp16"])
def test_block_against_the_oracle(T, d, f, operand):
    from paper_2303_11257_b200 import ffn
    host, b1, b2 = _make(T, d, f)
    dev = [torch.from_numpy(t).cuda() for t in host]
    block = ffn.UnitScaledBiasFFN(T, d, f, operand=operand, keep_h=True)
    block.b1.copy_(torch.from_numpy(b1))
    block.b2.copy_(torch.from_numpy(b2))
    block.step(*dev)
    block.check()
    sc = O.FFNScales.unconstrained(T, d, f)
    r, db1, db2 = O.bias_ffn_block(host[0], host[1], b1, host[2], b2, host[3], sc, operand)
    U.assert_close_stored(block.H, r.H, "bf16", 2e-3 * max(1.0, np.abs(r.H).max() / 4), "pre-activation")
    # (a column of few rows: one flipped code is a large part of it)
    for name, got, ref in (("A", block.Aq, r.Aq), ("dH", block.dHq, r.dHq), ("R", block.R, r.R), ("dW2", block.dW2, r.dW2), ("dW1", block.dW1, r.dW1), ("dX", block.dX, r.dX)):
        _near(got, ref, name, 1e-2 if operand == "fp8" else 4e-3)
    # the biases' gradients, from the gradients as the block holds them: (rows / 8 + 20) roundings of the sum of magnitudes
    for got, held in ((block.db1, block.dHq), (block.db2, block.Gq)):
        g = U.host_values(held)
        assert (np.abs(U.host_values(got) - O.bias_grad(g, sc.beta_w)) <= (T / 8 + 20) * 2.0 ** -24 * sc.beta_w * np.abs(g).sum(0)).all()
    _near(block.db1, db1, "db1", 2e-2 if operand == "fp8" else 4e-3)
    _near(block.db2, db2, "db2", 1e-5)
    # forward and backward on their own, and a step whose weights are in the operands already, do what a step does
    outs = lambda: [t.clone() for t in (block.R, block.dX, block.dW1, block.dW2, block.db1, block.db2)]
    want = outs()
    block.cast_weights(dev[1], dev[2])
    block.forward(dev[0])
    block.backward(dev[3])
    assert all(torch.equal(a, b) for a, b in zip(want, outs()))
    block.keep_h = False
    block.step(dev[0], None, None, dev[3])
    assert all(torch.equal(a, b) for a, b in zip(want, outs()))


@pytest.mark.parametrize("T,d,f,operand", [(256, 128, 512, "fp8"), (16000, 128, 400, "fp8"), (1000, 528, 2096, "bf16")])
def test_launches(T, d, f, operand):
    from paper_2303_11257_b200 import ffn, optim
    block = ffn.UnitScaledBiasFFN(T, d, f, operand=operand)
    X, W1, W2, G = (torch.zeros(s, device="cuda") for s in ((T, d), (d, f), (f, d), (T, d)))
    assert _kernels(lambda: block.step(X, W1, W2, G)) == block.launches_per_step == (5 if T == 16000 else 4)
    opt = optim.AdamW([W1, W2, block.b1, block.b2], [block.dW1, block.dW2, block.db1, block.db2], max_norm=1.0)
    assert _kernels(opt.step) == opt.launches_per_step == 2
    many = [torch.zeros(5, device="cuda") for _ in range(700)]
    opt = optim.AdamW(many, many, max_norm=1.0)
    assert _kernels(opt.step) == opt.launches_per_step == 5


@pytest.mark.parametrize("states", ["32bit", "8bit"])
@pytest.mark.parametrize("operand", ["fp8", "bf16"])
def test_training_steps(states, operand):
    """Steps of block and optimiser: every update is the oracle's from the gradients that the block left, the operands of the next step are the new weights, and a captured
    step does the same."""
    from paper_2303_11257_b200 import ffn, optim
    T, d, f = 200, 80, 208
    host, b1, b2 = _make(T, d, f)

    def build():
        X, W1, W2, G = (torch.from_numpy(t).cuda() for t in host)
        block = ffn.UnitScaledBiasFFN(T, d, f, operand=operand)
        block.cast_weights(W1, W2)
        params, grads = [W1, W2, block.b1, block.b2], [block.dW1, block.dW2, block.db1, block.db2]
        opt = optim.AdamW(params, grads, lr=0.02, weight_decay=[0.1, 0.1, 0.0, 0.0], copies=[block.W1q, block.W2q, None, None], states=states, max_norm=3.0)
        return X, G, block, opt
    X, G, block, opt = build()
    first = [p.clone() for p in opt.params]
    m = [np.zeros(p.numel()) for p in opt.params]
    v = [np.zeros(p.numel()) for p in opt.params]
    for t in range(1, 4):
        before = [U.host_values(p).ravel() for p in opt.params]
        block.step(X, None, None, G)
        opt.step()
        block.check()
        grads = [U.host_values(g).ravel() for g in opt.grads]
        norm, factor = O.grad_norm(grads, 3.0)
        assert abs(float(opt.norm[0]) - norm) <= 1e-6 * norm and abs(float(opt.norm[1]) - factor) <= 1e-6 * factor
        for i, (p, g, decay) in enumerate(zip(opt.params, grads, opt.weight_decay)):
            w = O.adamw_step(before[i], g, m[i], v[i], t, 0.02, weight_decay=decay, factor=factor)
            assert np.abs(U.host_values(p).ravel() - w.p).max() <= 2e-6 * np.abs(w.p).max(), (t, i)
            if states == "8bit":
                scale = lambda s: np.repeat(s.double().cpu().numpy(), 256)[:g.size]
                m[i] = scale(opt.m_scale[i]) * U.host_values(opt.m[i]).ravel()
                v[i] = (scale(opt.v_scale[i]) * U.host_values(opt.v[i]).ravel()) ** 2
                # half a step of E4M3 in its last binade, 16 of 448 = 0.0357 of a block's largest value; of v, (1 + 0.0357)^2 - 1 = 0.0727
                assert np.abs(m[i] - w.m).max() <= 0.0358 * np.abs(w.m).max() and np.abs(v[i] - w.v).max() <= 0.0728 * np.abs(w.v).max()
            else:
                m[i], v[i] = U.host_values(opt.m[i]).ravel(), U.host_values(opt.v[i]).ravel()
        for p, q in ((opt.params[0], block.W1q), (opt.params[1], block.W2q)):
            assert torch.equal(q.float(), p.clamp(-448, 448).to(q.dtype).float() if operand == "fp8" else p.to(q.dtype).float())
    assert opt.count.tolist() == [3, 0] and not any(torch.equal(a, b) for a, b in zip(first, opt.params))
    # the same steps, the last two of them replayed
    X2, G2, other, opt2 = build()
    other.step(X2, None, None, G2)
    opt2.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.step(X2, None, None, G2)
        opt2.step()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert opt2.count.tolist() == [3, 0] and all(torch.equal(a, b) for a, b in zip(opt.params, opt2.params))


def test_a_loss_of_one_block_has_the_gradients_of_differences():
    """db1, db2 of the block in FP16 against differences of its own forward pass: L = sum(R * G) along a direction of both biases.  Differences of 2^-4 in the biases; FP16 activations
    round by 2^-11 of themselves, with random signs over 64 x 96 outputs."""
    from paper_2303_11257_b200 import ffn
    T, d, f = 64, 96, 128
    host, b1, b2 = _make(T, d, f)
    X, W1, W2, G = (torch.from_numpy(t).cuda() for t in host)
    block = ffn.UnitScaledBiasFFN(T, d, f, operand="fp16", io_dtype=torch.float32, h_dtype=torch.float16)
    block.step(X, W1, W2, G)
    sc = block.sc
    rng = np.random.default_rng(5)
    u1, u2 = torch.from_numpy(rng.standard_normal(f)).float().cuda(), torch.from_numpy(rng.standard_normal(d)).float().cuda()
    branch = sc.tau ** 0.5
    slope1 = float((block.db1.double() * u1.double()).sum()) * branch / sc.beta_w * (sc.alpha2 / sc.beta_x2) * (sc.alpha_g / sc.beta_g)
    slope2 = float((block.db2.double() * u2.double()).sum()) * branch / sc.beta_w

    def loss(e1, e2):
        block.b1.copy_(e1 * u1)
        block.b2.copy_(e2 * u2)
        block.forward(X)
        return float((block.R.double() * G.double()).sum())
    h = 2.0 ** -4
    for slope, e in ((slope1, (h, 0.0)), (slope2, (0.0, h))):
        d_loss = (loss(*e) - loss(-e[0], -e[1])) / (2 * h)
        # rounding: 2^-12 of |A| ~ 1.7 in every product of a sum of T d f / f^(1/2) terms, times 1 / h; curvature: h^2 / 6 of a third derivative of the order of the slope's terms
        noise = 2.0 ** -12 * 2 * (T * d) ** 0.5 / h + h * h * (T * d) ** 0.5
        assert abs(d_loss - slope) <= 4 * noise, (d_loss, slope, noise)


def test_states_travel_to_another_optimiser():
    from paper_2303_11257_b200 import optim
    make = lambda: ([torch.randn(30, 50, device="cuda"), torch.randn(77, device="cuda")], [torch.randn(30, 50, device="cuda"), torch.randn(77, device="cuda")])
    p, g = make()
    for states in ("32bit", "8bit"):
        a = optim.AdamW([t.clone() for t in p], g, states=states)
        a.step()
        b = optim.AdamW([t.clone() for t in a.params], g, states=states)
        b.load_state_dict(a.state_dict())
        a.step()
        b.step()
        assert all(torch.equal(x, y) for x, y in zip(a.params, b.params)) and a.count.tolist() == b.count.tolist() == [2, 0]
    with pytest.raises(ValueError):
        b.load_state_dict(optim.AdamW(p, g).state_dict())


def test_calls_on_another_device_and_tensors_named_twice_are_refused(monkeypatch):
    from paper_2303_11257_b200 import lib as L
    from paper_2303_11257_b200 import optim
    p, q, g = (torch.ones(40, 64, device="cuda") for _ in range(3))
    opt, twice = optim.AdamW([p, q], [g, g], max_norm=1.0), optim.AdamW([p, p], [g, g])
    with pytest.raises(ValueError):
        twice.step()
    opt.step()
    before = p.clone()
    ws, out = L.new_workspace(), torch.empty(40, 64, dtype=torch.bfloat16, device="cuda")
    x = torch.ones(40, 64, device="cuda").bfloat16()
    monkeypatch.setattr(L, "_current_device", lambda: 7)
    for call in (opt.step, optim.AdamW([p], [g]).step, lambda: L.us_bias_grad([x], None, [q[0]]), lambda: L.us_linear_fwd_bias(x, x[:, :64], 1.0, q[0], out, ws)):
        with pytest.raises(ValueError):
            call()
    assert torch.equal(p, before) and opt.count.tolist() == [1, 0]


def test_other_tensors_are_laid_out_anew_and_lr_follows_the_schedule():
    from paper_2303_11257_b200 import optim
    p, g = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    factor = torch.ones(1, device="cuda")
    opt = optim.AdamW([p], [g], lr=0.5, weight_decay=0.0, lr_factor=factor)
    opt.step()
    assert torch.allclose(p, torch.full_like(p, 0.5))
    factor.fill_(0.5)
    opt.step()
    assert torch.allclose(p, torch.full_like(p, 0.25), atol=1e-5)
    opt.params[0] = q = torch.zeros(300, device="cuda")
    opt.step()
    assert torch.allclose(p, torch.full_like(p, 0.25), atol=1e-5) and torch.allclose(q, torch.full_like(q, -0.25), atol=1e-5)
    opt.weight_decay[0] = 1.0
    opt.lr = 0.1
    q.fill_(1.0)
    opt.step()
    assert torch.allclose(q, torch.full_like(q, 0.9), atol=1e-5)          # 1 - 0.05 (decay) - 0.05
