"""Windowed attention of rows: cases, references and the bounds that the kernels' roundings give."""
import numpy as np
import torch

from oracle import window_oracle as W

BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def half(dtype):
    return 2.0 ** -8 if dtype == BF16 else U


def reference(q, k, v, do, window, sinks, dtype, scale=None):
    """One head in fp64 -> {name: (value, bound)}.

    A score is a fp32 sum of D products of at most X in all, so off by (D + 16) U X, and the argument of its exponential
    by as much again and a rounding of itself; the normaliser likewise.  Probabilities and ds are rounded to the type
    for the second products (bf16: half a step; fp32: not at all), whose sums over L terms are fp32.  delta is formed
    from the rounded o."""
    n, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    o, lse, p = W.attention(q, k, v, window, sinks, scale)
    mask = W.sees(n, window, sinks)
    count = mask.sum(1).max()
    x = np.where(mask, scale * (np.abs(q) @ np.abs(k).T), 0).max()
    h, r = half(dtype), half(dtype) if dtype == BF16 else 0.0
    e = 4 * (d + 16) * U * x + (count + 64) * U + 8 * U * (1 + np.abs(lse).max())
    bo = h * np.abs(o) + (r + e) * (p @ np.abs(v))
    out = {"o": (o, bo), "lse": (lse, np.full(n, e))}
    if do is None:
        return out
    dq, dk, dv = W.gradients(q, k, v, do, window, sinks, scale)
    ds = np.where(mask, p * (do @ v.T - (do * o).sum(1)[:, None]), 0)
    off_dp = (d + 8) * U * (np.abs(do) @ np.abs(v).T)
    off_delta = (np.abs(do) * bo).sum(1) + (d + 8) * U * (np.abs(do) * np.abs(o)).sum(1)
    off = np.where(mask, np.abs(ds) * (r + e) + p * (1 + e) * (off_dp + off_delta[:, None]), 0)
    off = off * (1 + r) + (n + 64) * U * np.abs(ds)
    out["dq"] = dq, h * np.abs(dq) + scale * (off @ np.abs(k))
    out["dk"] = dk, h * np.abs(dk) + scale * (off.T @ np.abs(q))
    pe = (r + e + (n + 64) * U) * p
    out["dv"] = dv, h * np.abs(dv) + pe.T @ np.abs(do)
    return out


def grouped(q, k, v, do, window, sinks, dtype, scale=None):
    """[heads, n, D] and [kv_heads, n, D] -> the same of all heads, gradients of shared heads added up."""
    grp = len(q) // len(k)
    per = [reference(q[h], k[h // grp], v[h // grp], None if do is None else do[h], window, sinks, dtype, scale)
           for h in range(len(q))]
    out = {}
    for name in per[0]:
        if name in ("dk", "dv"):
            pick = lambda i: np.stack([sum(per[h][name][i] for h in range(a, a + grp)) for a in range(0, len(q), grp)])
        else:
            pick = lambda i: np.stack([x[name][i] for x in per])
        out[name] = pick(0), pick(1)
    return out


def check(name, got, want, bound):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), (name, "finite where it should be")
    ok = np.isfinite(want)
    err = np.abs(np.where(ok, got, 0) - np.where(ok, want, 0))
    bad = ok & ~(err <= bound + 1e-30)
    assert not bad.any(), (name, np.argwhere(bad)[:4], err[bad][:4], np.broadcast_to(bound, err.shape)[bad][:4])


def normal(rng, shape, dtype, scale=1.0):
    return (torch.from_numpy(rng.standard_normal(shape)) * scale).to(dtype)
