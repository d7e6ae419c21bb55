"""Plain fp64 statements of the operators around stage (b): final RMS norm, tied embedding, 8-bit
lm_head product, distillation from a teacher's top logits.  numpy, straight from the definitions;
shares no code with the CUDA library.  Used by the tests only."""
from __future__ import annotations

import numpy as np

NO_TOKEN = -1


# ---- final RMS norm ---------------------------------------------------------------------------
def rmsnorm_fwd(x, gamma, residual=None, eps=1e-6):
    """(s, rstd, h): s = x + residual, rstd = 1/sqrt(mean(s^2) + eps), h = s rstd gamma."""
    s = np.asarray(x, np.float64)
    if residual is not None:
        s = s + np.asarray(residual, np.float64)
    rstd = 1.0 / np.sqrt((s * s).mean(axis=1) + eps)
    return s, rstd, s * rstd[:, None] * np.asarray(gamma, np.float64)


def rmsnorm_bwd(dh, s, gamma, rstd, dsum=None):
    """(dx, dgamma) of h = s rstd gamma with rstd a function of s."""
    dh, s, gamma, rstd = (np.asarray(a, np.float64) for a in (dh, s, gamma, rstd))
    hat = s * rstd[:, None]
    gdh = dh * gamma
    dx = rstd[:, None] * (gdh - hat * (gdh * hat).mean(axis=1, keepdims=True))
    if dsum is not None:
        dx = dx + np.asarray(dsum, np.float64)
    return dx, (dh * hat).sum(axis=0)


def row_scales(h):
    """Scale of the 8-bit form of each row: max |h| / 127."""
    return np.abs(np.asarray(h, np.float64)).max(axis=1) / 127.0


# ---- tied embedding ---------------------------------------------------------------------------
def embed_fwd(W, y, scale=1.0):
    W = np.asarray(W, np.float64)
    X = np.zeros((len(y), W.shape[1]))
    for t, v in enumerate(np.asarray(y)):
        if 0 <= v < W.shape[0]:
            X[t] = scale * W[v]
    return X


def embed_bwd(dX, y, V, scale=1.0):
    """(dW, magnitude): dW[v] = scale sum_{y_t = v} dX_t, and the same sum of absolute values."""
    dX = np.asarray(dX, np.float64)
    dW = np.zeros((V, dX.shape[1]))
    mag = np.zeros((V, dX.shape[1]))
    ok = (np.asarray(y) >= 0) & (np.asarray(y) < V)
    np.add.at(dW, np.asarray(y)[ok], scale * dX[ok])
    np.add.at(mag, np.asarray(y)[ok], np.abs(scale * dX[ok]))
    return dW, mag


# ---- 8-bit lm_head product --------------------------------------------------------------------
def lmhead_q8(h8, h_scale, w8, w_scale):
    acc = np.asarray(h8, np.float64) @ np.asarray(w8, np.float64).T       # integers below 2^53: exact
    return acc * np.asarray(h_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64)[None, :]


# ---- distillation from a teacher's top logits ---------------------------------------------------
def teacher_probs(ids, logits, teacher_lse, V):
    """Row by row: log q of each list place (-inf for an empty one, or one whose logit is -inf or NaN)."""
    ids, logits = np.asarray(ids), np.asarray(logits, np.float64)
    there = (ids >= 0) & (ids < V)
    a = np.where(there & ~np.isnan(logits), logits, -np.inf)
    lq = np.full(a.shape, -np.inf)
    for t in range(len(a)):
        if not (a[t] > -np.inf).any():
            continue
        m = a[t].max()
        n = teacher_lse[t] if teacher_lse is not None else m + np.log(np.exp(a[t] - m).sum())
        lq[t] = a[t] - n
    return there, lq


def distill(H, W, ids, logits, cs, w, keep, teacher_lse=None, grad_scale=1.0):
    """loss = sum_t w_i sum_k q_tk (log q_tk - log p_t,id) over the rows of kept rollouts, and its gradients:
    dict of lse, kl, Q, mass (student's probability of the listed tokens, by list place), loss, dz, dH, dW."""
    H, W = np.asarray(H, np.float64), np.asarray(W, np.float64)
    T, V = H.shape[0], W.shape[0]
    cs = np.asarray(cs)
    owner = np.searchsorted(cs, np.arange(T), side="right") - 1
    kept = np.asarray(keep)[owner] != 0
    wt = np.asarray(w, np.float64)[owner] * kept
    z = H @ W.T
    m = z.max(axis=1, keepdims=True)
    lse = (m + np.log(np.exp(z - m).sum(axis=1, keepdims=True)))[:, 0]
    there, lq = teacher_probs(ids, logits, teacher_lse, V)
    at = np.where(there, ids, 0).astype(np.int64)
    q = np.exp(lq)
    lp = np.take_along_axis(z, at, axis=1) - lse[:, None]
    with np.errstate(invalid="ignore"):
        kl = np.where(q > 0, q * (lq - lp), 0.0).sum(axis=1) * kept
    Q = q.sum(axis=1)
    dz = Q[:, None] * np.exp(z - lse[:, None])
    for t in range(T):
        np.add.at(dz[t], at[t], -q[t])
    dz *= (grad_scale * wt)[:, None]
    return dict(lse=lse * kept, kl=kl, Q=Q, q=q, lq=lq, lp=lp, there=there, kept=kept, wt=wt, z=z, loss=float((wt * kl).sum()),
                dz=dz, dH=dz @ W, dW=dz.T @ H, mass=np.where(there, np.exp(lp), 0.0).sum(axis=1))
