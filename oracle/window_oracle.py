"""Plain fp64 reference of causal attention with a sliding window and sinks, of its gradients, and of rotary positions.

Test infrastructure only: the package does not import it and it imports nothing from the package.  NumPy, one sequence
and head at a time, straight from the formulas.
"""
import numpy as np


def sees(n, window, sinks):
    """[n, n]: token i sees token j."""
    i, j = np.arange(n)[:, None], np.arange(n)[None]
    return (j <= i) & ((j < sinks) | (j > i - window))


def attention(q, k, v, window, sinks, scale=None):
    """q, k, v [n, D] -> (o [n, D], lse [n], p [n, n]).  What a token does not see is not touched."""
    n, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    mask = sees(n, window, sinks)
    o, lse, p = np.zeros_like(q), np.zeros(n), np.zeros((n, n))
    for i in range(n):
        j = np.nonzero(mask[i])[0]
        with np.errstate(invalid="ignore", over="ignore"):
            s = scale * (k[j] @ q[i])
            m = s.max()
            lse[i] = m + np.log(np.exp(s - m).sum())
            p[i, j] = np.exp(s - lse[i])
            o[i] = p[i, j] @ v[j]
    return o, lse, p


def gradients(q, k, v, do, window, sinks, scale=None):
    """(dq, dk, dv) of sum(do * o)."""
    n, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    mask = sees(n, window, sinks)
    o, _, p = attention(q, k, v, window, sinks, scale)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for i in range(n):
        j = np.nonzero(mask[i])[0]
        with np.errstate(invalid="ignore", over="ignore"):
            ds = p[i, j] * (v[j] @ do[i] - do[i] @ o[i])
            dq[i] = scale * (ds @ k[j])
            dk[j] += scale * ds[:, None] * q[i]
            dv[j] += p[i, j][:, None] * do[i]
    return dq, dk, dv


def rotate(x, pos, axis, freq, halves=False, inverse=False):
    """x [tokens, ..., D] turned by pos [tokens, axes]: axis, freq [D / 2], axis -1: the pair stays."""
    half = x.shape[-1] // 2
    y = x.copy()
    for j in range(half):
        if axis[j] < 0:
            continue
        a, b = (j, j + half) if halves else (2 * j, 2 * j + 1)
        phi = pos[:, axis[j]].astype(np.float64) * freq[j] * (-1 if inverse else 1)
        phi = phi.reshape((-1,) + (1,) * (x.ndim - 2))
        c, s = np.cos(phi), np.sin(phi)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y
