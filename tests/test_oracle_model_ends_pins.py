"""Pins of the fp64 statements of the operators around stage (b): scalar loops, autograd of an
independent torch statement, finite differences.  CPU only."""
import math

import numpy as np
import pytest
import torch

from oracle import model_ends as M


@pytest.mark.parametrize("with_residual", [False, True])
def test_rmsnorm_against_scalar_loops_and_autograd(with_residual):
    rng = np.random.default_rng(3)
    T, d, eps = 4, 7, 1e-3
    x, r, gamma, dh, dsum = (rng.standard_normal(s) for s in ((T, d), (T, d), d, (T, d), (T, d)))
    s, rstd, h = M.rmsnorm_fwd(x, gamma, r if with_residual else None, eps)
    for t in range(T):
        row = [x[t, k] + (r[t, k] if with_residual else 0.0) for k in range(d)]
        rms = math.sqrt(sum(v * v for v in row) / d + eps)
        for k in range(d):
            assert h[t, k] == pytest.approx(row[k] / rms * gamma[k], rel=1e-13)
    xt, gt = torch.tensor(s, requires_grad=True), torch.tensor(gamma, requires_grad=True)
    ht = xt * torch.rsqrt(xt.square().mean(1, keepdim=True) + eps) * gt
    ((ht * torch.tensor(dh)).sum() + (xt * torch.tensor(dsum)).sum()).backward()
    dx, dgamma = M.rmsnorm_bwd(dh, s, gamma, rstd, dsum)
    assert np.allclose(dx, xt.grad.numpy(), rtol=1e-12, atol=1e-14)
    assert np.allclose(dgamma, gt.grad.numpy(), rtol=1e-12, atol=1e-14)


def test_rmsnorm_gradient_against_differences():
    rng = np.random.default_rng(4)
    T, d, eps, step = 2, 5, 1e-2, 1e-6
    x, gamma, dh = rng.standard_normal((T, d)), rng.standard_normal(d), rng.standard_normal((T, d))
    s, rstd, _ = M.rmsnorm_fwd(x, gamma, None, eps)
    dx, dgamma = M.rmsnorm_bwd(dh, s, gamma, rstd)
    f = lambda a, g: float((M.rmsnorm_fwd(a, g, None, eps)[2] * dh).sum())
    for t in range(T):
        for k in range(d):
            e = np.zeros_like(x)
            e[t, k] = step
            assert dx[t, k] == pytest.approx((f(x + e, gamma) - f(x - e, gamma)) / (2 * step), rel=1e-6, abs=1e-8)
    for k in range(d):
        e = np.zeros(d)
        e[k] = step
        assert dgamma[k] == pytest.approx((f(x, gamma + e) - f(x, gamma - e)) / (2 * step), rel=1e-6, abs=1e-8)


def test_embedding_against_autograd():
    rng = np.random.default_rng(5)
    V, d, T = 6, 3, 11
    W, dX = rng.standard_normal((V, d)), rng.standard_normal((T, d))
    y = rng.integers(0, V, T)
    y[[2, 7]] = M.NO_TOKEN
    Wt = torch.tensor(W, requires_grad=True)
    X = 1.5 * torch.nn.functional.embedding(torch.tensor(np.where(y < 0, V, y)), torch.cat([Wt, torch.zeros(1, d)]))
    assert np.allclose(M.embed_fwd(W, y, 1.5), X.detach().numpy(), rtol=1e-14)
    (X * torch.tensor(dX)).sum().backward()
    dW, mag = M.embed_bwd(dX, y, V, 1.5)
    assert np.allclose(dW, Wt.grad.numpy(), rtol=1e-13, atol=1e-15)
    assert (mag >= np.abs(dW) - 1e-15).all()


def test_8bit_product_by_scalar_loops():
    rng = np.random.default_rng(6)
    h8, w8 = rng.integers(-128, 128, (3, 16)), rng.integers(-128, 128, (5, 16))
    sh, sw = rng.random(3), rng.random(5)
    z = M.lmhead_q8(h8, sh, w8, sw)
    for t in range(3):
        for v in range(5):
            assert z[t, v] == pytest.approx(sum(int(a) * int(b) for a, b in zip(h8[t], w8[v])) * sh[t] * sw[v], rel=1e-14)


def _distill_case(seed=0, T=9, d=5, V=12, K=4):
    rng = np.random.default_rng(seed)
    H, W = rng.standard_normal((T, d)), rng.standard_normal((V, d))
    ids = np.stack([rng.choice(V, K, replace=False) for _ in range(T)])
    logits = rng.standard_normal((T, K)) * 2
    ids[1, 2:] = M.NO_TOKEN
    ids[2] = M.NO_TOKEN
    ids[3, 1] = ids[3, 0]                       # a token listed twice
    logits[4, 0] = -np.inf
    cs, keep, w = np.array([0, 3, 5, T]), np.array([1, 0, 1]), np.array([0.3, 0.0, 0.2])
    return H, W, ids, logits, cs, w, keep


@pytest.mark.parametrize("given_lse", [False, True])
def test_distillation_against_autograd_of_its_definition(given_lse):
    H, W, ids, logits, cs, w, keep = _distill_case(1)
    tl = np.full(len(H), 3.0) if given_lse else None
    got = M.distill(H, W, ids, logits, cs, w, keep, tl, grad_scale=1.3)
    Ht, Wt = torch.tensor(H, requires_grad=True), torch.tensor(W, requires_grad=True)
    logp = torch.log_softmax(Ht @ Wt.T, dim=1)
    loss = 0.0
    for i in range(3):
        for t in range(cs[i], cs[i + 1] if keep[i] else cs[i]):
            place = [k for k in range(ids.shape[1]) if ids[t, k] >= 0 and logits[t, k] > -np.inf]
            a = torch.tensor([logits[t, k] for k in place], dtype=torch.float64)
            lq = a - (tl[t] if given_lse else torch.logsumexp(a, 0)) if place else a
            for j, k in enumerate(place):
                loss = loss + w[i] * torch.exp(lq[j]) * (lq[j] - logp[t, ids[t, k]])
    (1.3 * loss).backward()
    assert got["loss"] == pytest.approx(loss.item(), rel=1e-12)
    assert np.allclose(got["dH"], Ht.grad.numpy(), rtol=1e-10, atol=1e-13)
    assert np.allclose(got["dW"], Wt.grad.numpy(), rtol=1e-10, atol=1e-13)
    assert got["kl"][2] == 0 and not got["dH"][2].any() and not got["dH"][3:5].any() and not got["lse"][3:5].any()


def test_distillation_gradient_against_differences():
    H, W, ids, logits, cs, w, keep = _distill_case(2)
    got = M.distill(H, W, ids, logits, cs, w, keep)
    step = 1e-6
    for t, k in ((0, 0), (1, 3), (5, 2), (8, 4)):
        e = np.zeros_like(H)
        e[t, k] = step
        f = lambda s: M.distill(H + s * e, W, ids, logits, cs, w, keep)["loss"]
        assert got["dH"][t, k] == pytest.approx((f(1) - f(-1)) / (2 * step), rel=1e-5, abs=1e-9)
    for v, k in ((0, 1), (7, 4), (11, 0)):
        e = np.zeros_like(W)
        e[v, k] = step
        f = lambda s: M.distill(H, W + s * e, ids, logits, cs, w, keep)["loss"]
        assert got["dW"][v, k] == pytest.approx((f(1) - f(-1)) / (2 * step), rel=1e-5, abs=1e-9)


def test_distillation_from_the_policy_itself_is_at_its_minimum():
    """The whole vocabulary listed with the student's own logits: kl = 0 and no gradient; columns of dW sum to 0."""
    H, W, _, _, cs, w, keep = _distill_case(3)
    z = H @ W.T
    got = M.distill(H, W, np.tile(np.arange(len(W)), (len(H), 1)), z, cs, w, keep)
    assert np.abs(got["kl"]).max() < 1e-12 and np.abs(got["dH"]).max() < 1e-12
    ids, logits = _distill_case(3)[2:4]
    assert np.abs(M.distill(H, W, ids, logits, cs, w, keep)["dW"].sum(axis=0)).max() < 1e-12
