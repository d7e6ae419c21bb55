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
