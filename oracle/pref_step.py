"""Plain fp64 statements of the operators of a preference-training step: the loss on pairs of rollouts, the AdamW step with its
8-bit states, rows in 4-bit floating point.  numpy, straight from the definitions; shares no code with the CUDA library.
Used by the tests only."""
from __future__ import annotations

import numpy as np

NO_TOKEN = -1


# ---- preference loss on pairs of rollouts ---------------------------------------------------------
def pref_pair(kind, m, smoothing=0.0):
    """(loss, slope) of a margin."""
    if kind == "logistic":
        sig = lambda x: np.exp(-np.logaddexp(0.0, -x))  # noqa: E731
        return ((1 - smoothing) * np.logaddexp(0.0, -m) + smoothing * np.logaddexp(0.0, m),
                smoothing * sig(m) - (1 - smoothing) * sig(-m))
    if kind == "square":
        return (m - 0.5) ** 2, 2 * (m - 0.5)
    return max(0.0, 1.0 - m), -1.0 if m < 1 else 0.0


def preference(H, W, y, cs, pairs, ref=None, weight=None, kind="logistic", mean=False, beta=0.1, margin=0.0, smoothing=0.0,
               grads=True):
    """Outputs of the loss on pairs by its definition; rows of rollouts in no pair are 0."""
    H, W = np.asarray(H, np.float64), np.asarray(W, np.float64)
    T, V, R = len(H), len(W), len(cs) - 1
    counted = [p for p, (c, r) in enumerate(pairs) if 0 <= c < R and 0 <= r < R]
    used = sorted({i for p in counted for i in pairs[p]})
    logp, lse = np.zeros(T), np.zeros(T)
    ratio, coef = np.zeros(R), np.zeros(R)
    scored = {i: [t for t in range(cs[i], cs[i + 1]) if 0 <= y[t] < V] for i in used}
    for i in used:
        for t in range(cs[i], cs[i + 1]):
            z = W @ H[t]
            lse[t] = z.max() + np.log(np.exp(z - z.max()).sum())
        for t in scored[i]:
            logp[t] = W[y[t]] @ H[t] - lse[t]
        ratio[i] = sum(logp[t] - (0.0 if ref is None else float(ref[t])) for t in scored[i])
        if mean and scored[i]:
            ratio[i] /= len(scored[i])
    m = np.zeros(len(pairs))
    loss = 0.0
    for p in counted:
        c, r = pairs[p]
        u = 1.0 / len(counted) if weight is None else float(weight[p])
        m[p] = beta * (ratio[c] - ratio[r]) - margin
        each, slope = pref_pair(kind, m[p], smoothing)
        loss += u * each
        for i, sign in ((c, 1.0), (r, -1.0)):
            coef[i] += sign * u * beta * slope / (len(scored[i]) if mean and scored[i] else 1)
    n = max(1, len(counted))
    out = dict(logp=logp, lse=lse, ratio=ratio, margin=m, coef=coef, loss=loss,
               metrics=np.array([sum(ratio[pairs[p][0]] > ratio[pairs[p][1]] for p in counted) / n,
                                 beta * sum(ratio[pairs[p][0]] for p in counted) / n,
                                 beta * sum(ratio[pairs[p][1]] for p in counted) / n, len(counted)]))
    if grads:
        dz = np.zeros((T, V))
        for i in used:
            for t in scored[i]:
                dz[t] = -coef[i] * np.exp(W @ H[t] - lse[t])
                dz[t, y[t]] += coef[i]
        out.update(dz=dz, dH=dz @ W, dW=dz.T @ H)
    return out


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


# ---- rows in 4-bit floating point -----------------------------------------------------------------
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_to(x, table):
    """The nearest value of a table of magnitudes (its last one for what is larger), the one at an even place of two as near."""
    a = np.minimum(np.abs(x), table[-1])
    hi = np.clip(np.searchsorted(table, a), 1, len(table) - 1)
    below, above = a - table[hi - 1], table[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return np.sign(x) * np.where(up, table[hi], table[hi - 1])


def quantize_fp4(x, block):
    """(values, scales of the blocks, row scales or None) of rows x."""
    x = np.asarray(x, np.float64)
    T, d = x.shape
    xb = x.reshape(T, d // block, block)
    top = np.abs(xb).max(axis=2)
    if block == 32:
        m, e = np.frexp(top)                                   # top = m 2^e, m in [0.5, 1)
        scale, row = np.ldexp(1.0, np.where(top > 0, np.maximum(e - 3, -127), -127)), None
    else:
        m, e = np.frexp(np.abs(x).max(axis=1) / (6 * 448))
        row = np.where(m > 0, np.ldexp(1.0, np.maximum(e - (m == 0.5), -126)), 0.0)
        unit = np.where(row > 0, row, 1.0)
        scale = round_to(top / 6 / unit[:, None], E4M3) * row[:, None]
    safe = np.where(scale > 0, scale, 1.0)
    value = round_to(xb / safe[:, :, None], E2M1) * scale[:, :, None]
    return value.reshape(T, d), scale, row


def fp4_places(T, d, block):
    """Byte and half of each code, and byte of each scale, in the library's layout."""
    slabs = -(-d // 256)
    r, c = np.arange(T)[:, None], np.arange(d)[None, :]
    byte = c % 256 // 2
    at = ((r // 128 * slabs + c // 256) * 128 + r % 128) * 128 + ((byte // 16) ^ (r % 8)) * 16 + byte % 16
    k = np.arange(d // block)[None, :]
    groups = slabs * 64 // block
    return at, c % 2 + 0 * r, (r // 128 * groups + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4


def fp4_values(codes, scales, row, T, d, block):
    """The values that buffers in that layout hold."""
    at, half, where = fp4_places(T, d, block)
    code = (codes[at] >> (4 * half)) & 15
    s = scales[where].astype(np.int64)
    if block == 32:
        scale = np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    else:
        scale = np.concatenate([E4M3, [np.nan]])[s & 127] * np.asarray(row, np.float64)[:, None]
    return np.where(code >= 8, -1.0, 1.0) * E2M1[code & 7] * np.repeat(scale, block, axis=1)
