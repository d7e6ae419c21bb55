"""Plain fp64 statements of the operators of a preference-training step: the loss on pairs of rollouts, the AdamW step with its
8-bit states, rows in 4-bit floating point.  numpy, straight from the definitions; shares no code with the CUDA library.
Used by the tests only."""
from __future__ import annotations

import numpy as np

NO_TOKEN = -1


# ---- AdamW ------------------------------------------------------------------------------------
E4M3 = np.array([(8 * (c > 7) + c % 8) * 2.0 ** (max(c // 8, 1) - 10) for c in range(127)])          # magnitudes of codes 0 .. 126
E4M4 = np.array([(16 * (c > 15) + c % 16) * 2.0 ** (max(c // 16, 1) - 11) for c in range(256)])


def grad_norm(grads, grad_scale=1.0):
    return abs(grad_scale) * np.sqrt(sum((np.asarray(g, np.float64) ** 2).sum() for g in grads))


def clip_of(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6)) if max_norm > 0 else 1.0


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, factor=1.0):
    """(p, m, v) after step t; factor = grad_scale * clip."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = g * factor
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    step = (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return (1 - lr * weight_decay) * p - lr * step, m, v


def blocks_of(x, size=256):
    """x in rows of `size`, zeros behind the end."""
    x = np.asarray(x, np.float64).ravel()
    return np.concatenate([x, np.zeros(-len(x) % size)]).reshape(-1, size)


def state_scales(m, v):
    """Scales per 256 elements of m and of the root of v."""
    least = 2.0 ** -100
    return (np.maximum(np.abs(blocks_of(m)).max(1), least) / 448, np.maximum(np.sqrt(blocks_of(v)).max(1), least) / 496)


def nearest(x, table):
    """Distance of each x from the nearest value of a table."""
    at = np.clip(np.searchsorted(table, x), 1, len(table) - 1)
    return np.minimum(np.abs(x - table[at - 1]), np.abs(table[at] - x))
