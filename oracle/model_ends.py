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
