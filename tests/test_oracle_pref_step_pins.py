"""Pins of the fp64 statements of a preference-training step: hand values, differences, an independent torch statement.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import pref_step as M


def case(seed, T=23, d=5, V=11):
    g = np.random.default_rng(seed)
    H, W = g.normal(size=(T, d)), g.normal(size=(V, d))
    y = g.integers(0, V, T)
    y[[4, 9]] = M.NO_TOKEN
    return H, W, y, [0, 6, 6, 11, 17, 23], [(0, 2), (0, 3), (2, 3), (-1, -1), (3, 3), (1, 0), (7, 0)], g.normal(size=T), g.random(7)


@pytest.mark.parametrize("kind", ["logistic", "square", "hinge"])
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
def test_preference_against_autograd_and_differences(kind, mean, weighted):
    H, W, y, cs, pairs, ref, weight = case(1)
    kw = dict(kind=kind, mean=mean, beta=0.4, margin=0.1, smoothing=0.2, weight=weight if weighted else None)
    out = M.preference(H, W, y, cs, pairs, ref, **kw)
    h, w = torch.tensor(H, requires_grad=True), torch.tensor(W, requires_grad=True)
    lp = torch.log_softmax(h @ w.T, 1)
    ok = torch.tensor(y >= 0)
    lp = torch.where(ok, lp[torch.arange(len(y)), torch.tensor(y).clamp(min=0)] - torch.tensor(ref), torch.zeros(()).double())
    n = [max(1, int(ok[a:b].sum())) if mean else 1 for a, b in zip(cs, cs[1:])]
    r = torch.stack([lp[a:b].sum() / k for a, b, k in zip(cs, cs[1:], n)])
    live = [p for p, q in enumerate(pairs) if min(q) >= 0 and max(q) < 5]
    m = torch.stack([0.4 * (r[pairs[p][0]] - r[pairs[p][1]]) - 0.1 for p in live])
    if kind == "logistic":
        each = -0.8 * torch.nn.functional.logsigmoid(m) - 0.2 * torch.nn.functional.logsigmoid(-m)
    elif kind == "square":
        each = (m - 0.5) ** 2
    else:
        each = torch.relu(1 - m)
    u = torch.tensor(weight)[live] if weighted else torch.full((len(live),), 1 / len(live), dtype=torch.float64)
    loss = (u * each).sum()
    loss.backward()
    assert abs(out["loss"] - loss.item()) < 1e-12
    assert np.abs(out["dH"] - h.grad.numpy()).max() < 1e-12 and np.abs(out["dW"] - w.grad.numpy()).max() < 1e-12
    for t, k in ((0, 1), (7, 3), (16, 0), (20, 2)):
        d = np.zeros_like(H)
        d[t, k] = 1e-6
        up, down = (M.preference(H + s * d, W, y, cs, pairs, ref, grads=False, **kw)["loss"] for s in (1, -1))
        assert abs((up - down) / 2e-6 - out["dH"][t, k]) < 1e-8
    assert not out["dH"][17:].any() and not out["logp"][17:].any()          # the fifth rollout is in no pair that counts
    assert out["metrics"][3] == len(live)


def test_preference_by_hand():
    """Two tokens, a vocabulary of two, weights that give probabilities 3/4 and 1/4."""
    W, H = np.array([[np.log(3.0)], [0.0]]), np.ones((2, 1))
    out = M.preference(H, W, [0, 1], [0, 1, 2], [(0, 1)], beta=1.0)
    m = np.log(3.0)                                                    # log(3/4) - log(1/4)
    assert np.allclose(out["ratio"], [np.log(0.75), np.log(0.25)]) and np.isclose(out["margin"][0], m)
    assert np.isclose(out["loss"], np.log(4 / 3)) and np.allclose(out["coef"], [-0.25, 0.25])
    assert np.allclose(out["dz"], [[-0.25 * 0.25, 0.25 * 0.25], [-0.25 * 0.75, 0.25 * 0.75]])


def test_adamw_against_torch():
    g = np.random.default_rng(2)
    p, grads = g.normal(size=40), g.normal(size=(4, 40))
    ref = torch.nn.Parameter(torch.tensor(p))
    opt = torch.optim.AdamW([ref], lr=0.05, betas=(0.8, 0.97), eps=1e-6, weight_decay=0.3)
    m, v = np.zeros(40), np.zeros(40)
    for t in range(4):
        ref.grad = torch.tensor(grads[t])
        total = torch.nn.utils.clip_grad_norm_([ref], 2.0).item()
        assert np.isclose(total, M.grad_norm([grads[t]]))
        opt.step()
        p, m, v = M.adamw(p, grads[t], m, v, t + 1, 0.05, 0.8, 0.97, 1e-6, 0.3, M.clip_of(total, 2.0))
        assert np.allclose(p, ref.detach().numpy(), rtol=1e-12, atol=1e-12)


def test_eight_bit_tables():
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(M.E4M3, e4m3)
    assert M.E4M4[0] == 0 and M.E4M4[1] == 2.0 ** -10 and M.E4M4[16] == 2.0 ** -6 and M.E4M4[255] == 496
    assert np.all(np.diff(M.E4M4) > 0) and np.all(np.diff(M.E4M4)[16:] / M.E4M4[16:-1] <= 1 / 16)
    ms, vs = M.state_scales(np.array([0.0] * 300), np.array([4.0] * 256 + [0.0] * 44))
    assert np.all(ms == 2.0 ** -100 / 448) and vs[0] == 2 / 496 and vs[1] == 2.0 ** -100 / 496


def test_four_bit_rows_by_hand():
    x = np.zeros((2, 32))
    x[0, :8] = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25]
    value, scale, row = M.quantize_fp4(x, 32)
    assert scale[0, 0] == 1 and list(value[0, :8]) == [6, 4, 4, 2, 2, 1, 1, 0] and not value[1].any()
    value, scale, row = M.quantize_fp4(x * 448, 16)
    assert row[0] == 1 and scale[0, 0] == 448 and list(value[0, :8]) == [448 * v for v in (6, 4, 4, 2, 2, 1, 1, 0)]
    assert row[1] == 0 and scale[1, 0] == 0 and scale[0, 1] == 0
    x[0, :2] = [7.9, -8]
    value, scale, _ = M.quantize_fp4(x, 32)
    assert scale[0, 0] == 2 and list(value[0, :2]) == [8, -8]
    x[0, :2] = [7.9, -7.9]
    assert list(M.quantize_fp4(x, 32)[0][0, :2]) == [6, -6]               # beyond 6: 6


def test_places_of_four_bit_rows_are_a_layout():
    for T, d, block in ((130, 288, 16), (5, 32, 32), (129, 544, 32)):
        at, half, where = M.fp4_places(T, d, block)
        assert len(set(zip(at.ravel(), half.ravel()))) == T * d and len(set(where.ravel())) == T * (d // block)
        assert at.max() < -(-T // 128) * -(-d // 256) * 128 * 128 and where.max() < -(-T // 128) * -(-d // 256) * 128 * 256 // block
