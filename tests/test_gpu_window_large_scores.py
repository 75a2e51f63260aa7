"""Gradients of the windowed attention where scores are so large that an fp32 log-sum-exp no longer holds them: a
probability does not pass 1 by more than that rounding, and not at all where it is large, so finite inputs have finite
gradients."""
import numpy as np
import pytest
import torch

from oracle import window_oracle as W

from _window import BF16, F32, U, check, half, normal

pytestmark = pytest.mark.gpu


def within(name, got, most):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), (name, np.argwhere(~np.isfinite(got))[:4])
    bad = ~(np.abs(got) <= most)
    assert not bad.any(), (name, np.argwhere(bad)[:4], got[bad][:4], most[bad][:4])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("exponent", [5, 10, 12, 14, 20, 24, 27, 35, 60, 100])
@pytest.mark.parametrize("n,window,sinks", [(200, 70, 5), (300, 280, 0)])     # the second: two groups of waves share tiles
def test_probabilities_stay_below_one(dtype, d, exponent, n, window, sinks):
    """Scores are multiples of 2^exponent.  With 0 <= p <= 1
      |dv_j| <= sum_i |do_i|,  |ds_ij| <= |do_i| |v_j| + |do_i| |o_i|,  |dq_i| <= sum_j |ds_ij| |k_j|,
    and dk likewise, whose delta is corrected by the row's sum of ds, at most that of its bounds.  The bounds count the
    roundings of p, ds and the results (three half steps) and of n + 2 d fp32 operations.  p itself is bounded by 1 for
    rows whose log-sum-exp passes 2^20 (to base 2); below, it may pass 1 by what that is off: the largest score times
    its constant, the sum with log2 l, to base e and back are six roundings, log2 l another."""
    from paper_2605_15684_amd import window as mod
    rng = np.random.default_rng(d + exponent)
    q, k = torch.zeros(1, 1, n, d, dtype=dtype), torch.zeros(1, 1, n, d, dtype=dtype)
    rank = rng.permutation(256)[:n] if n <= 256 else np.arange(n) % 256      # 8 bits: exact in bf16
    q[..., 7] = 2.0 ** exponent
    k[..., 7] = torch.from_numpy(rank + 1.0).to(dtype)
    v, do = normal(rng, (1, 1, n, d), dtype), normal(rng, (1, 1, n, d), dtype)
    kw = dict(window=window, sinks=sinks, scale=1.0)
    dev = [x.cuda() for x in (q, k, v, do)]
    o, lse = mod.forward(*dev[:3], **kw)
    dq, dk, dv = mod.backward(*dev[:3], o, dev[3], lse, **kw)
    torch.cuda.synchronize()
    q, k, v, do, o = (np.abs(x[0, 0].double().cpu().numpy()) for x in (q, k, v, do, o))
    mask = W.sees(n, window, sinks)
    base2 = float(lse.abs().max()) * 1.4427
    more = (1 + half(dtype)) ** 3 * (1 + (n + 2 * d + 64) * U) * 2 ** (6 * U * min(base2, 2.0 ** 20) + 2.0 ** -20)
    ds = np.where(mask, do @ v.T + (do * o).sum(1)[:, None], 0)
    off = ds.sum(1)                                         # what the corrected delta may differ by
    within("dv", dv[0, 0], more * (mask.T @ do) + 1e-30)
    within("dq", dq[0, 0], more * (ds @ k) + 1e-30)
    within("dk", dk[0, 0], more * (np.where(mask, ds + off[:, None], 0).T @ q) + 1e-30)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_of_large_terms_that_cancel(dtype):
    """Products of up to 2^60 whose sum is small: a score is off by the rounding of its terms, far more than exp2 takes."""
    from paper_2605_15684_amd import window as mod
    rng = np.random.default_rng(1)
    n, d = 150, 64
    q, k, v, do = (normal(rng, (1, 2, n, d), dtype) for _ in range(4))
    q[..., 3] = 2.0 ** 30
    q[..., 40] = -2.0 ** 30
    k[..., 3] = k[..., 40] = (k[..., 3].abs() + 1) * 2.0 ** 30
    kw = dict(window=60, sinks=2, scale=1.0)
    dev = [x.cuda() for x in (q, k, v, do)]
    o, lse = mod.forward(*dev[:3], **kw)
    grads = mod.backward(*dev[:3], o, dev[3], lse, **kw)
    for name, x in zip(("o", "dq", "dk", "dv"), (o,) + grads):
        assert torch.isfinite(x).all(), name
    # The scores are the forward's, on both sides: only what the log-sum-exp is off by takes p past 1.
    more = (1 + half(dtype)) ** 3 * (1 + (n + 64) * U) * 2 ** (6 * U * min(float(lse.abs().max()) * 1.4427, 2.0 ** 20) + 2.0 ** -20)
    most = torch.from_numpy(W.sees(n, 60, 2).T.astype(np.float64)) @ do[0].abs().double()
    assert (grads[2][0].double().cpu().abs() <= most * more).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_large_rows_beside_ordinary_ones(dtype, d):
    """Rows of 2^24 times larger scores among ordinary ones, keys that both see: dq of the ordinary rows, and dv where
    the large rows' probabilities are 0 or 1 whatever the rounding, within the bounds of exact scores."""
    from _window import reference
    from paper_2605_15684_amd import window as mod
    rng = np.random.default_rng(d)
    n, window = 200, 40
    q, k, v, do = (normal(rng, (1, 1, n, d), dtype) for _ in range(4))
    large = np.arange(n) % 50 == 17
    q[0, 0, large] = 0
    q[0, 0, large, 5] = 2.0 ** 24
    do[0, 0, large] = 0                          # the large rows pass nothing back: every gradient is that of the others
    dev = [x.cuda() for x in (q, k, v, do)]
    o, lse = mod.forward(*dev[:3], window=window)
    dq, dk, dv = mod.backward(*dev[:3], o, dev[3], lse, window=window)
    small = q.clone()
    small[0, 0, large] = 0
    ref = reference(*(x[0, 0].double().numpy() for x in (small, k, v, do)), window, 0, dtype)
    for name, x in (("dq", dq), ("dk", dk), ("dv", dv)):
        check(name, x[0, 0], *ref[name])


def test_a_nan_that_is_seen_still_reaches_every_gradient():
    """Bounding a probability from above does not turn a NaN score into a number."""
    from paper_2605_15684_amd import window as mod
    rng = np.random.default_rng(2)
    n, d = 140, 64
    for dtype in (BF16, F32):
        q, k, v, do = (normal(rng, (1, 1, n, d), dtype) for _ in range(4))
        q[0, 0, 50, 9] = float("nan")
        dev = [x.cuda() for x in (q, k, v, do)]
        o, lse = mod.forward(*dev[:3], window=20)
        dq, dk, dv = mod.backward(*dev[:3], o, dev[3], lse, window=20)
        seen = W.sees(n, 20, 0)[50]
        assert torch.isnan(dq[0, 0, 50]).all() and torch.isfinite(dq[0, 0, torch.arange(n) != 50]).all()
        for x in (dk, dv):
            assert torch.isnan(x[0, 0, torch.from_numpy(seen)]).all() and torch.isfinite(x[0, 0, torch.from_numpy(~seen)]).all()
