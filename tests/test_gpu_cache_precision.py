"""How precisely the cache's attention holds its probabilities, in every form of its kernel.

Bound of a value, with W = sum_j p_j |v_j| and E of tests/test_gpu_cache.py (scores and sums in fp32):

  half |o| + (u + E) W + a

half: half a step of the output.  u: what a probability loses, 2^-16 as two bf16 terms (each is off by at most 2^-8 of
what it holds), 2^-11 in fp16, 2^-22 in fp32.  a: fp16 has steps of 2^-24 below 2^-14, and the largest probability times
its page's V scale is held at 2^8 or more, so that a weight is off by at most 2^-33 of the largest one: 2^-33 * 448 *
L * (largest V scale) over all keys."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as C

from _cache import gpu_batch, gpu_pool, make_batch, make_pool, rounded

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

FORMS = [  # page, D, heads, kv heads, keep (0: the whole sequence), bits of a bf16 call's probabilities, sequences
    (16, 64, 4, 2, 0, 16, [(250, 1), (90, 1)]),               # up to 16 columns: 4 waves
    (16, 128, 16, 2, 0, 16, [(1000, 2), (700, 1)]),           # 8 waves
    (32, 64, 8, 2, 0, 16, [(5000, 1)]),                       # parts that are joined
    (16, 64, 10, 2, 0, 11, [(200, 4), (130, 2)]),             # 32 columns: 4 waves
    (64, 128, 10, 2, 0, 11, [(1000, 4), (300, 6)]),           # 8 waves
    (16, 128, 10, 2, 0, 11, [(4000, 4)]),                     # parts
    (16, 64, 10, 2, 0, 11, [(240, 8), (40, 7)]),              # 64 columns
    (32, 128, 10, 2, 0, 11, [(3000, 8)]),
    (16, 64, 20, 2, 0, 11, [(250, 10), (233, 9)]),            # 128
    (32, 128, 20, 2, 0, 11, [(3000, 10)]),
    (16, 64, 6, 2, 0, 11, [(400, 100), (300, 37)]),           # 256
    (64, 128, 6, 2, 0, 11, [(2500, 100)]),
    (16, 64, 4, 2, 5, 16, [(300, 2), (120, 1)]),              # lists: 4 waves to a row
    (32, 128, 16, 2, 40, 16, [(2000, 2)]),                    # 8 waves
    (64, 64, 8, 2, 50, 16, [(4000, 1)]),                      # parts
    (16, 64, 16, 16, 3, 11, [(300, 130)]),                    # a wave to a row, two shares of its keys
    (16, 128, 128, 16, 3, 11, [(300, 130)]),
    (16, 64, 192, 16, 3, 11, [(250, 130)]),                   # the same, more than 8 query heads to a kv head
]


def check(got, ref, length, d, dtype, bits, most_v):
    o, w, x = ref
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    u = 2.0 ** -bits if dtype == BF16 else 2.0 ** -22
    e = 4 * (d + 16) * 2.0 ** -24 * x[..., None] + (length + 64) * 2.0 ** -24
    a = 2.0 ** -33 * 448 * length * most_v if dtype == BF16 and bits == 11 else 0.0
    err = np.abs(got.double().cpu().numpy() - o)
    bound = half * np.abs(o) + (u + e) * w + a + 1e-30
    bad = ~(err <= bound)
    assert not bad.any(), (np.argwhere(bad)[:4], err[bad][:4], bound[bad][:4])


def some_lists(rng, seqs, kv, keep, page):
    """Distinct pages of what each token sees, its own last one among them."""
    out = []
    for held, new in seqs:
        for r in range(new):
            own = (held - new + r) // page
            for _ in range(kv):
                n = min(keep, own + 1)
                ids = np.sort(np.append(rng.permutation(own)[:n - 1], own))
                out.append(np.concatenate([[n], ids, np.full(keep - n, -1)]))
    return np.array(out, dtype=np.int32).reshape(-1, kv, 1 + keep)


def run(pool, batch, q, lists, seqs, scale=None):
    from paper_2605_15684_amd import cache
    b = gpu_batch(batch, max(n for _, n in seqs), max(h for h, _ in seqs))
    return cache.attend(gpu_pool(pool), 0, b, q.cuda(), scale=scale,
                        lists=None if lists is None else torch.from_numpy(lists).cuda())


@pytest.mark.parametrize("page,d,heads,kv,keep,bits,seqs", FORMS)
def test_attend_bits_of_the_probabilities(page, d, heads, kv, keep, bits, seqs):
    """Every second key has the weight 0.50191, which bf16 rounds to 0.5, and a value of -2 against 1: the outputs nearly
    cancel, and what the rounding of all these weights changes does not."""
    rng = np.random.default_rng(1)
    pages, rows = sum(-(-h // page) for h, _ in seqs), sum(n for _, n in seqs)
    pool = make_pool(rng, 1, pages, kv, d, page)
    ko, vo = C.orders(page, d)
    one, minus_one, minus_two = C.e4m3([1.0, -1.0, -2.0])
    pool["k"][:] = 0
    pool["k"][..., ko[1::2, 0]] = minus_one
    pool["v"][..., vo[0::2].ravel()] = one
    pool["v"][..., vo[1::2].ravel()] = minus_two
    pool["scale"][:] = 1.0
    batch = make_batch(rng, seqs, page, pages)
    q = torch.zeros(rows, heads, d, dtype=BF16)
    q[..., 0] = 1.0
    lists = some_lists(rng, seqs, kv, keep, page) if keep else None
    scale = float(np.float32(-math.log(0.5 + 0.98 * 2.0 ** -9)))
    got = run(pool, batch, q, lists, seqs, scale)
    ref = C.attend(pool, 0, batch, q.double().numpy(), page, lists, True, scale)
    length = keep * page if keep else max(h for h, _ in seqs)
    check(got, ref, length, d, BF16, bits, 1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,d,heads,kv,keep,bits,seqs", FORMS)
def test_attend_scores_that_outgrow_the_maximum(page, d, heads, kv, keep, bits, seqs, dtype):
    """Scores that grow along the sequence by hundreds, up and down between: the maximum is raised again and again, the
    last pages weigh the most; V's scales differ by up to 2^18 from page to page."""
    rng = np.random.default_rng(2)
    pages, rows = sum(-(-h // page) for h, _ in seqs), sum(n for _, n in seqs)
    pool = make_pool(rng, 1, pages, kv, d, page)
    batch = make_batch(rng, seqs, page, pages)
    for s, (held, _) in enumerate(seqs):
        ids = batch[0][s][: -(-held // page)]
        grow = np.linspace(-10, -4, len(ids)) + rng.uniform(-1, 1, len(ids))
        pool["scale"][0, ids, :, 0] = (2.0 ** grow.round()).astype(np.float32)[:, None]
    pool["scale"][..., 1] = (2.0 ** rng.integers(-12, 7, pool["scale"].shape[:3])).astype(np.float32)
    q, q64 = rounded(rng, (rows, heads, d), dtype, 2.0)
    lists = some_lists(rng, seqs, kv, keep, page) if keep else None
    got = run(pool, batch, q, lists, seqs)
    ref = C.attend(pool, 0, batch, q64, page, lists)
    length = keep * page if keep else max(h for h, _ in seqs)
    check(got, ref, length, d, dtype, bits, 64.0)


@pytest.mark.parametrize("page,d,heads,kv,keep,bits,seqs", FORMS)
def test_attend_queries_that_are_nan(page, d, heads, kv, keep, bits, seqs):
    """A query with a NaN makes its own output NaN and leaves all others as precise as they are."""
    rng = np.random.default_rng(3)
    pages, rows = sum(-(-h // page) for h, _ in seqs), sum(n for _, n in seqs)
    pool = make_pool(rng, 1, pages, kv, d, page)
    batch = make_batch(rng, seqs, page, pages)
    q, q64 = rounded(rng, (rows, heads, d), BF16, 0.3)
    lists = some_lists(rng, seqs, kv, keep, page) if keep else None
    o, w, x = C.attend(pool, 0, batch, q64, page, lists)
    bad = rng.random((rows, heads)) < 0.2
    bad[0, 0] = True
    bad[-1, -1] = False
    q[torch.from_numpy(bad)] = torch.where(torch.arange(d) == 5, float("nan"), q[torch.from_numpy(bad)].float()).to(BF16)
    got = run(pool, batch, q, lists, seqs).float().cpu().numpy()
    assert np.isnan(got[bad]).all()
    length = keep * page if keep else max(h for h, _ in seqs)
    check(torch.from_numpy(np.where(bad[..., None], o, got)), (o, w, x), length, d, BF16, bits, 2.0 ** -6)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,d,heads,kv,keep,bits,seqs", FORMS)
def test_attend_scales_of_every_size(page, d, heads, kv, keep, bits, seqs, dtype):
    """V's scales from the smallest that append writes to 2^60, powers of two and others, in pages of one sequence; then
    the smallest alone.  A page of 2^60 outweighs the others, as it does in W."""
    rng = np.random.default_rng(4)
    pages, rows = sum(-(-h // page) for h, _ in seqs), sum(n for _, n in seqs)
    batch = make_batch(rng, seqs, page, pages)
    q, q64 = rounded(rng, (rows, heads, d), dtype, 0.5)
    lists = some_lists(rng, seqs, kv, keep, page) if keep else None
    length = keep * page if keep else max(h for h, _ in seqs)
    for sizes in ([2.0 ** -64, 1.7 * 2.0 ** -40, 1.0, 0.6, 2.0 ** 60], [2.0 ** -64, 1.3 * 2.0 ** -64]):
        pool = make_pool(rng, 1, pages, kv, d, page)
        pool["scale"][..., 0] *= rng.uniform(0.5, 1.0, pool["scale"].shape[:3]).astype(np.float32)
        pool["scale"][..., 1] = rng.choice(sizes, pool["scale"].shape[:3]).astype(np.float32)
        got = run(pool, batch, q, lists, seqs)
        check(got, C.attend(pool, 0, batch, q64, page, lists), length, d, dtype, bits, max(sizes))
