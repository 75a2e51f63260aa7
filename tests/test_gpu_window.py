"""Causal attention with a sliding window and sinks on the GPU, forward and backward, against the fp64 oracle
(oracle/window_oracle.py).  Tolerances: the sum of the roundings that the kernels make (tests/_window.py)."""
import numpy as np
import pytest
import torch

from oracle import window_oracle as W

from _window import BF16, F32, check, grouped, normal

pytestmark = pytest.mark.gpu


def run(q, k, v, do, **kw):
    from paper_2605_15684_amd import window
    o, lse = window.forward(q, k, v, **kw)
    out = {"o": o, "lse": lse}
    if do is not None:
        out["dq"], out["dk"], out["dv"] = window.backward(q, k, v, o, do, lse, **kw)
    torch.cuda.synchronize()
    return out


BATCHES = [  # batch, heads, kv heads, D, rows, window, sinks, dtype
    (1, 1, 1, 64, 1, 1, 0, BF16),
    (2, 2, 1, 128, 1, 5, 3, F32),
    (1, 2, 2, 128, 2, 1, 1, BF16),
    (1, 3, 1, 64, 31, 7, 0, BF16),
    (1, 2, 1, 128, 33, 100, 4, F32),
    (2, 4, 2, 128, 65, 32, 1, BF16),
    (1, 2, 2, 64, 127, 64, 70, BF16),
    (1, 1, 1, 64, 128, 128, 0, F32),
    (1, 6, 2, 64, 129, 64, 5, F32),
    (1, 4, 1, 128, 200, 33, 130, BF16),
    (3, 8, 8, 64, 150, 16, 2, BF16),
    (1, 2, 1, 64, 300, 2147483647, 2147483647, BF16),
    (1, 2, 1, 128, 257, 1, 0, F32),
    (1, 1, 1, 64, 1300, 40, 3, BF16),      # the queries of the sinks in two chunks
    (1, 2, 1, 128, 1100, 100, 130, F32),   # two such tiles
]


@pytest.mark.parametrize("b,h,kv,d,n,window,sinks,dtype", BATCHES)
def test_batch(b, h, kv, d, n, window, sinks, dtype):
    rng = np.random.default_rng(n + d)
    q, do = (normal(rng, (b, h, n, d), dtype) for _ in range(2))
    k, v = (normal(rng, (b, kv, n, d), dtype) for _ in range(2))
    got = run(*(t.cuda() for t in (q, k, v, do)), window=window, sinks=sinks)
    for x in range(b):
        ref = grouped(*(t[x].double().numpy() for t in (q, k, v, do)), window, sinks, dtype)
        for name, (want, bound) in ref.items():
            check(name, got[name][x], want, bound)


PACKED = [  # lengths, heads, kv heads, D, window, sinks, dtype
    ([1], 1, 1, 64, 3, 1, BF16),
    ([5, 0, 130, 1, 64], 4, 2, 128, 50, 4, BF16),
    ([0, 0, 200, 0], 2, 1, 64, 64, 0, F32),
    ([128, 128, 1, 127, 300], 2, 2, 64, 100, 140, BF16),
    ([33, 2, 97], 6, 2, 128, 17, 2, F32),
    ([1, 1200, 77, 1030], 2, 1, 64, 90, 5, BF16),      # chunks of two sequences, none of the others
]


@pytest.mark.parametrize("lens,h,kv,d,window,sinks,dtype", PACKED)
def test_packed(lens, h, kv, d, window, sinks, dtype):
    rng = np.random.default_rng(sum(lens) + d)
    before, behind = 3, 5                        # rows of no sequence
    rows = before + sum(lens) + behind
    q, do = (normal(rng, (rows, h, d), dtype) for _ in range(2))
    k, v = (normal(rng, (rows, kv, d), dtype) for _ in range(2))
    nan = torch.tensor(float("nan"), dtype=dtype)
    for t in (q, k, v, do):
        t[:before] = nan
        t[rows - behind:] = nan
    at = before + np.concatenate([[0], np.cumsum(lens)])
    cu = torch.from_numpy(at.astype(np.int32)).cuda()
    from paper_2605_15684_amd import window as mod
    dev = [t.cuda() for t in (q, k, v, do)]
    kw = dict(window=window, sinks=sinks, cu=cu)
    mark = 7.0
    o, dq = (torch.full_like(dev[0], mark) for _ in range(2))
    dk, dv = (torch.full_like(dev[1], mark) for _ in range(2))
    lse = torch.full((h, rows), mark, device="cuda")
    mod.forward(*dev[:3], **kw, out=o, lse=lse)
    mod.backward(*dev[:3], o, dev[3], lse, **kw, dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    for s, n in enumerate(lens):
        if not n:
            continue
        rowset = slice(at[s], at[s] + n)
        ref = grouped(*(t[rowset].double().numpy().transpose(1, 0, 2) for t in (q, k, v, do)), window, sinks, dtype)
        for name, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
            check(name, t[rowset].transpose(0, 1), *ref[name])
        check("lse", lse[:, rowset], *ref["lse"])
    for t in (o, dq, dk, dv, lse.T):
        assert (t[:before] == mark).all() and (t[rows - behind:] == mark).all(), "rows of no sequence were written"
    # the hint about lengths does not change results
    for hint in (1, max(lens), 10 ** 6):
        again = mod.forward(*dev[:3], **kw, max_len=hint)
        assert torch.equal(again[0][at[0]:at[-1]], o[at[0]:at[-1]])


def test_scores_that_outgrow_the_running_maximum():
    """Keys grow along the row, so that the maximum is raised again and again, by more than 2^20 each time."""
    rng = np.random.default_rng(5)
    for dtype in (BF16, F32):
        n, d = 400, 64
        q, do = normal(rng, (1, 1, n, d), dtype), normal(rng, (1, 1, n, d), dtype)
        k = (torch.ones(1, 1, n, d) * torch.linspace(0, 40, n)[:, None]).to(dtype)
        q = (q.abs() * 0.5).to(dtype)
        v = normal(rng, (1, 1, n, d), dtype)
        got = run(*(t.cuda() for t in (q, k, v, do)), window=200, sinks=3)
        ref = grouped(*(t[0].double().numpy() for t in (q, k, v, do)), 200, 3, dtype)
        for name, (want, bound) in ref.items():
            check(name, got[name][0], want, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("exponent", [5, 20, 35])
def test_scores_past_what_exp2_takes(dtype, d, exponent):
    """Scores of distinct multiples of 2^exponent, exact in fp32: the largest takes all, to the last bit; those behind
    it are at most exp(-32) of it, together 2^-45."""
    rng = np.random.default_rng(d + exponent)
    n, window, sinks = 200, 70, 5
    q, k = torch.zeros(1, 1, n, d, dtype=dtype), torch.zeros(1, 1, n, d, dtype=dtype)
    rank = rng.permutation(n).astype(np.int64) + 1          # up to 8 bits: exact in bf16
    q[..., 7] = 2.0 ** exponent
    k[..., 7] = torch.from_numpy(rank).to(dtype)
    v = normal(rng, (1, 1, n, d), dtype)
    got = run(q.cuda(), k.cuda(), v.cuda(), None, window=window, sinks=sinks, scale=1.0)
    for i in range(n):
        seen = [j for j in range(i + 1) if j < sinks or j > i - window]
        best = max(seen, key=lambda j: rank[j])
        want = v[0, 0, best].double().numpy()
        # o = (p v) (1 / p).  bf16: p and the result are rounded.  fp32: six products of terms in turn, three left out
        # of 2^-24 each, 1 / p, the product.
        bound = (11 * 2.0 ** -24 if dtype == F32 else 2 * 2.0 ** -8) * np.abs(want) + 2.0 ** -36
        assert np.all(np.abs(got["o"][0, 0, i].double().cpu().numpy() - want) <= bound), i
        # To base 2 and back: two constants, three operations, and the logarithm of p.
        assert abs(float(got["lse"][0, 0, i]) / (2.0 ** exponent * rank[best]) - 1) <= 6 * 2.0 ** -24, i


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_hidden_places_hold_anything(dtype, d):
    """NaN and infinities in single rows of one input at a time: what does not see them keeps its result."""
    rng = np.random.default_rng(d)
    n, window, sinks, h = 260, 50, 3, 2
    base = [normal(rng, (1, x, n, d), dtype) for x in (h, 1, 1, h)]
    bad = [float("nan"), float("inf"), float("-inf")]
    for which in range(4):
        for case, row in enumerate((0, 1, 40, 130, 255)):
            t = [x.clone() for x in base]
            t[which][0, 0, row, case * 7 % d] = bad[(which + case) % 3]
            got = run(*(x.cuda() for x in t), window=window, sinks=sinks)
            ref = grouped(*(x[0].double().numpy() for x in t), window, sinks, dtype)
            for name, (want, bound) in ref.items():
                # bounds of rows that see the value are not finite; those rows only have to be as finite as the result
                check(name, got[name][0], want, np.where(np.isfinite(bound), bound, np.inf))


SHARED = [  # few rows of long windows: the tiles of a workgroup go to two groups of waves
    (1, 2, 1, 64, 600, 300, 5, F32),
    (2, 2, 2, 64, 390, 390, 0, BF16),
    (1, 4, 2, 128, 520, 260, 130, BF16),
    (1, 2, 1, 64, 300, 250, 6, F32),
    (1, 2, 1, 128, 257, 500, 0, BF16),
    (1, 2, 1, 64, 1500, 257, 2, BF16),     # queries of the sinks in chunks
]


@pytest.mark.parametrize("b,h,kv,d,n,window,sinks,dtype", SHARED)
def test_shared_tiles(b, h, kv, d, n, window, sinks, dtype):
    test_batch(b, h, kv, d, n, window, sinks, dtype)


@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (64, F32)])
def test_hidden_places_of_shared_tiles(d, dtype):
    """As test_hidden_places_hold_anything: a group of waves that sees the value computes once more, and the other."""
    rng = np.random.default_rng(d + 1)
    n, window, sinks, h = 400, 256, 3, 2
    base = [normal(rng, (1, x, n, d), dtype) for x in (h, 1, 1, h)]
    bad = [float("nan"), float("inf"), float("-inf")]
    for which in range(4):
        for case, row in enumerate((2, 70, 300)):
            t = [x.clone() for x in base]
            t[which][0, 0, row, case * 7 % d] = bad[(which + case) % 3]
            got = run(*(x.cuda() for x in t), window=window, sinks=sinks)
            ref = grouped(*(x[0].double().numpy() for x in t), window, sinks, dtype)
            for name, (want, bound) in ref.items():
                check(name, got[name][0], want, np.where(np.isfinite(bound), bound, np.inf))


def test_strides():
    """q, k and v as views of one projection's output, outputs into views too."""
    from paper_2605_15684_amd import window
    rng = np.random.default_rng(9)
    b, n, h, kv, d = 2, 140, 4, 2, 64
    for dtype in (BF16, F32):
        proj = normal(rng, (b, n, h + 2 * kv, d), dtype).cuda()
        q, k, v = (x.transpose(1, 2) for x in proj.split([h, kv, kv], 2))
        do = normal(rng, (b, h, n, d), dtype).cuda()
        grads = torch.zeros_like(proj)
        dq, dk, dv = (x.transpose(1, 2) for x in grads.split([h, kv, kv], 2))
        out = torch.empty((b, n, h, d), dtype=dtype, device="cuda").transpose(1, 2)
        kw = dict(window=60, sinks=2, scale=0.2)
        o, lse = window.forward(q, k, v, out=out, **kw)
        window.backward(q, k, v, o, do, lse, dq=dq, dk=dk, dv=dv, **kw)
        want = run(*(x.contiguous() for x in (q, k, v)), do, **kw)
        for x, name in ((o, "o"), (lse, "lse"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
            assert torch.equal(x, want[name]), name
        ref = grouped(*(x[0].double().cpu().numpy() for x in (q, k, v, do)), 60, 2, dtype, 0.2)
        for name, (value, bound) in ref.items():
            check(name, want[name][0], value, bound)


@pytest.mark.parametrize("h,kv,d,n,window,sinks,dtype", [
    (2, 2, 64, 500, 200, 5, F32), (3, 1, 128, 300, 130, 0, F32), (2, 1, 64, 333, 64, 140, F32), (1, 1, 128, 700, 511, 3, F32),
    (2, 2, 128, 900, 600, 2, BF16), (1, 1, 64, 1500, 100, 130, F32)])
def test_shared_queries(h, kv, d, n, window, sinks, dtype):
    """Few tiles: several workgroups share the queries of each, and the heads."""
    test_batch(1, h, kv, d, n, window, sinks, dtype)


@pytest.mark.parametrize("d", [64, 128])
def test_shared_queries_of_packed_sequences(d):
    """Shares of sequences of any length, of which short ones leave most shares without a query."""
    test_packed([1, 400, 0, 33, 128], 2, 1, d, 300, 2, F32)
