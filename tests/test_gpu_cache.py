"""The paged 8-bit cache on the GPU against the fp64 oracle
(oracle/cache_oracle.py).

Append, select and the page calls are compared exactly (codes, scales, pooled
keys, lists, tables).  Attention is compared within

  bf16: 2^-8 |o| + (2^-8 + E) W        fp32: 2^-24 |o| + (2^-22 + E) W
  W = sum_j p_j |v_j|,  E = 4 (D + 16) 2^-24 X + (L + 64) 2^-24,  X = max_j scale sum |q k_j|

half a step of the output; half a step of each probability (bf16 rounds them
once, fp32 holds 24 bits in three terms); E: a score is a sum of D products in
fp32, whose error turns into a relative one of its probability and of the
normaliser, and sums over the L keys."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C

from _cache import assert_same_pool, gpu_batch, gpu_pool, host_pool, make_batch, make_pool, rounded

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def check_attend(got, ref, length, d, dtype):
    o, w, x = ref
    rows = ~np.isnan(o[:, :, 0])
    half, p = (2.0 ** -8, 2.0 ** -8) if dtype == BF16 else (2.0 ** -24, 2.0 ** -22)
    e = 4 * (d + 16) * 2.0 ** -24 * x[..., None] + (length + 64) * 2.0 ** -24
    err = np.abs(got.double().cpu().numpy() - o)
    bound = half * np.abs(o) + (p + e) * w + 1e-30
    bad = ~(err <= bound) & rows[..., None]
    assert not bad.any(), (np.argwhere(bad)[:4], err[bad][:4], bound[bad][:4])


# ---- append -------------------------------------------------------------------

APPENDS = [  # page, D, kv heads, dtype, sequences (held, new)
    (64, 128, 2, BF16, [(1, 1)]),
    (64, 128, 4, BF16, [(64, 1), (65, 1), (130, 130), (63, 0), (191, 64)]),
    (16, 64, 3, F32, [(77, 77), (16, 16), (15, 2), (33, 18)]),
    (32, 64, 1, BF16, [(100, 3), (64, 33), (31, 31)]),
    (16, 128, 5, BF16, [(48, 47), (49, 1), (50, 20)]),
    (32, 128, 2, F32, [(95, 95), (96, 1), (97, 2)]),
    (64, 64, 1, F32, [(128, 65), (127, 1)]),
]


@pytest.mark.parametrize("page,d,kv,dtype,seqs", APPENDS)
def test_append(page, d, kv, dtype, seqs):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(page + d + kv)
    rows, pages = sum(n for _, n in seqs), sum(-(-h // page) for h, _ in seqs) + 2
    pool = make_pool(rng, 2, pages, kv, d, page)
    batch = make_batch(rng, seqs, page, pages)
    scale = 10.0 ** rng.uniform(-3, 1.5, (rows, 1, 1))
    k, k64 = rounded(rng, (rows, kv, d), dtype, torch.from_numpy(scale))
    v, v64 = rounded(rng, (rows, kv, d), dtype, torch.from_numpy(scale[::-1].copy()))
    gpool = gpu_pool(pool)
    cache.append(gpool, 1, gpu_batch(batch, max(n for _, n in seqs)), k.cuda(), v.cuda())
    C.append(pool, 1, batch, k64, v64, page)
    assert_same_pool(host_pool(gpool), pool)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_token_by_token(dtype):
    """Scales that grow within a page: older codes are restated, step by step like the oracle's."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(7)
    page, d, kv, n = 32, 64, 2, 70
    pool = make_pool(rng, 1, 4, kv, d, page)
    gpool = gpu_pool(pool)
    table = np.array([[3, 0, 1]], dtype=np.int32)
    k, k64 = rounded(rng, (n, kv, d), dtype, torch.from_numpy(2.0 ** rng.uniform(-6, 6, (n, 1, 1))))
    v, v64 = rounded(rng, (n, kv, d), dtype, torch.from_numpy(2.0 ** rng.uniform(-6, 6, (n, 1, 1))))
    at = 0
    while at < n:
        m = min(int(rng.integers(1, 4)), n - at)
        batch = (table, np.array([at + m], dtype=np.int32), np.array([0, m], dtype=np.int32))
        cache.append(gpool, 0, gpu_batch(batch, m), k[at:at + m].cuda(), v[at:at + m].cuda())
        C.append(pool, 0, batch, k64[at:at + m], v64[at:at + m], page)
        at += m
    assert_same_pool(host_pool(gpool), pool)


def test_append_extreme_values():
    """NaN, infinities, zeros, the smallest and largest numbers; a page of infinities alone."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(8)
    page, d, kv, n = 16, 64, 1, 64
    k, _ = rounded(rng, (n, kv, d), F32)
    k[3, 0, 5], k[4, 0, 6], k[5, 0, 7] = float("nan"), float("inf"), -float("inf")
    k[16:32] = float("inf")
    k[32:48] = 0.0
    k[33, 0, 1], k[34, 0, 1] = 1e-45, -1e-38
    k[48, 0, 0], k[49, 0, 1], k[50], k[51, 0, 3] = 3.4028234e38, -3.4028234e38, 1e30, float("inf")
    v = -k
    pool = make_pool(rng, 1, 4, kv, d, page)
    gpool = gpu_pool(pool)
    batch = (np.array([[2, 1, 0, 3]], dtype=np.int32), np.array([n], dtype=np.int32), np.array([0, n], dtype=np.int32))
    cache.append(gpool, 0, gpu_batch(batch, n), k.cuda(), v.cuda())
    with np.errstate(all="ignore"):
        C.append(pool, 0, batch, k.double().numpy(), v.double().numpy(), page)
    assert_same_pool(host_pool(gpool), pool)


def test_append_strided_and_offset_rows():
    """K and V as slices of a fused projection; rows of no sequence in front and behind."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(9)
    page, d, kv = 16, 64, 2
    pool = make_pool(rng, 1, 6, kv, d, page)
    qkv, qkv64 = rounded(rng, (30, 8, d), BF16)
    table, lens, cu = make_batch(rng, [(20, 20), (18, 3)], page, 6)
    cu = cu + 4
    g = qkv.cuda()
    gpool = gpu_pool(pool)
    cache.append(gpool, 0, gpu_batch((table, lens, cu), 20), g[:, 4:6], g[:, 6:8])
    C.append(pool, 0, (table, lens, cu), qkv64[:, 4:6], qkv64[:, 6:8], page)
    assert_same_pool(host_pool(gpool), pool)


def test_append_passes_over_what_is_not_there():
    """Pages out of range, a sequence shorter than its new rows, rows past the array, an idle sequence."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(10)
    page, d, kv = 16, 64, 1
    pool = make_pool(rng, 1, 6, kv, d, page)
    gpool = gpu_pool(pool)
    table = np.array([[0, -1, 99, 1], [2, 3, -1, -1], [4, 5, -1, -1], [4, 5, -1, -1]], dtype=np.int32)
    lens = np.array([60, 5, 1 << 30, 20], dtype=np.int32)      # the third is cut to the table
    cu = np.array([0, 40, 50, 70, 90], dtype=np.int32)
    lens[2] = 10 ** 9
    x, x64 = rounded(rng, (80, kv, d), BF16)
    cache.append(gpool, 0, gpu_batch((table, lens, cu), 40), x.cuda(), x.cuda())
    lens_cut = lens.copy()
    C.append(pool, 0, (table, lens_cut, cu), x64, x64, page)
    assert_same_pool(host_pool(gpool), pool)


# ---- attend ---------------------------------------------------------------------

ATTENDS = [  # page, D, heads, kv heads, dtype, causal, sequences
    (64, 64, 1, 1, BF16, True, [(1, 1)]),
    (64, 64, 4, 1, BF16, True, [(4096, 1)]),
    (64, 128, 16, 4, BF16, True, [(1, 1), (64, 1), (65, 1), (1000, 1), (333, 0), (32, 1)]),
    (16, 128, 6, 2, BF16, True, [(17, 1), (16, 1), (15, 1), (500, 1)]),
    (32, 64, 40, 2, BF16, True, [(100, 1), (31, 1)]),                     # 20 query heads to a kv head
    (16, 64, 6, 2, BF16, True, [(40, 9), (9, 9), (200, 3)]),              # two column tiles a wave
    (64, 128, 16, 4, BF16, True, [(1000, 8), (300, 5), (2, 2)]),          # the same, 8 waves
    (16, 64, 16, 4, BF16, False, [(5000, 7)]),                            # in parts
    (32, 128, 8, 2, BF16, False, [(300, 12), (12, 12), (77, 1)]),         # four
    (64, 128, 4, 2, BF16, True, [(200, 130), (70, 70), (300, 64)]),       # by columns
    (16, 64, 3, 1, BF16, False, [(333, 100), (22, 22)]),
    (16, 64, 12, 4, BF16, True, [(3000, 20), (40, 17), (333, 5)]),        # 64 columns, keys shared by 8 waves and split
    (32, 128, 8, 2, BF16, False, [(2000, 25), (60, 32)]),                 # 128 columns, keys split
    (64, 64, 6, 1, BF16, True, [(1500, 90), (600, 600)]),                 # tiles of 256 columns
    (16, 64, 8, 4, BF16, True, [(300, 300), (700, 150), (129, 129), (400, 5)]),   # the same, heads a multiple of 8
    (16, 64, 16, 8, BF16, True, [(2000, 40)]),                            # and keys split
    (64, 128, 5, 1, F32, True, [(1, 1), (700, 1)]),
    (64, 128, 5, 1, F32, True, [(2900, 2), (700, 3)]),
    (16, 64, 6, 2, F32, False, [(1500, 4), (3, 3), (0, 0)]),
    (32, 64, 4, 2, F32, True, [(5000, 1)]),
    (16, 64, 6, 2, F32, True, [(50, 7), (7, 7), (129, 2)]),
    (32, 128, 4, 2, F32, False, [(150, 60), (64, 33)]),
]


@pytest.mark.parametrize("page,d,heads,kv,dtype,causal,seqs", ATTENDS)
def test_attend(page, d, heads, kv, dtype, causal, seqs):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(page + d + heads + len(seqs))
    pages, rows = sum(-(-h // page) for h, _ in seqs) + 3, sum(n for _, n in seqs)
    pool = make_pool(rng, 2, pages, kv, d, page)
    batch = make_batch(rng, seqs, page, pages)
    # what lies behind the ends and in other pages is NaN
    used = np.zeros(pages, dtype=bool)
    for s, (held, _) in enumerate(seqs):
        ids = batch[0][s][: -(-held // page)]
        used[ids] = True
        if held % page:
            for which, x in enumerate("kv"):
                pool[x][1, ids[-1]][:, C.orders(page, d)[which][held % page:].ravel()] = 127
    for x in "kv":
        pool[x][1, ~used] = 255
    pool["scale"][1, ~used] = np.nan
    q, q64 = rounded(rng, (rows, heads, d), dtype, 0.2)
    g = gpu_pool(pool)
    got = cache.attend(g, 1, gpu_batch(batch, max(n for _, n in seqs), max(h for h, _ in seqs)), q.cuda(), causal=causal)
    check_attend(got, C.attend(pool, 1, batch, q64, page, causal=causal), max(h for h, _ in seqs), d, dtype)


@pytest.mark.parametrize("max_len", [None, 1, 300, 100000])
def test_attend_whatever_the_length_hint(max_len):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(11)
    page, d, heads, kv, seqs = 16, 64, 4, 2, [(900, 1), (3, 1), (450, 1)]
    pool = make_pool(rng, 1, 100, kv, d, page)
    batch = make_batch(rng, seqs, page, 100, spare=7)
    q, q64 = rounded(rng, (3, heads, d), BF16, 0.2)
    got = cache.attend(gpu_pool(pool), 0, gpu_batch(batch, 1, max_len), q.cuda())
    check_attend(got, C.attend(pool, 0, batch, q64, page), 900, d, BF16)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attend_strides_scale_and_rows_left_alone(new, dtype):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(12)
    page, d, heads, kv = 32, 64, 6, 3
    seqs = [(50, new), (90, new)]
    pool = make_pool(rng, 1, 8, kv, d, page)
    table, lens, cu = make_batch(rng, seqs, page, 8)
    cu = cu + 2
    rows = int(cu[-1]) + 3
    qkv, qkv64 = rounded(rng, (rows, 12, d), dtype, 0.3)
    out = torch.full((rows, 8, d), 5.0, dtype=dtype, device="cuda")
    got = cache.attend(gpu_pool(pool), 0, gpu_batch((table, lens, cu), new), qkv.cuda()[:, 3:9], scale=0.37,
                       out=out[:, 1:7])
    ref = C.attend(pool, 0, (table, lens, cu), qkv64[:, 3:9], page, scale=0.37)
    check_attend(got, ref, 90, d, dtype)
    rest = out.clone()
    rest[2:int(cu[-1]), 1:7] = 5.0
    assert (rest == 5.0).all()


def test_attend_large_scores():
    """Scores that keep growing along the sequence by hundreds: the maximum is raised again and again."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(13)
    page, d, heads, kv = 16, 64, 4, 2
    pool = make_pool(rng, 1, 80, kv, d, page)
    batch = make_batch(rng, [(600, 1), (600, 5)], page, 80)
    q, q64 = rounded(rng, (6, heads, d), F32, 3.0)
    for s in range(2):
        ids = batch[0][s][:38]
        pool["scale"][0, ids, :, 0] = (2.0 ** np.linspace(-9, -3, 38).round()).astype(np.float32)[:, None]
    got = cache.attend(gpu_pool(pool), 0, gpu_batch(batch, 5), q.cuda())
    check_attend(got, C.attend(pool, 0, batch, q64, page), 600, d, F32)


@pytest.mark.parametrize("new", [1, 6, 30])
def test_attend_pages_that_are_not_there(new):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(14)
    page, d, heads, kv = 16, 64, 4, 1
    pool = make_pool(rng, 1, 10, kv, d, page)
    table, lens, cu = make_batch(rng, [(80, new), (45, new), (30, new)], page, 10, spare=2)
    pool["v"][0, 0] = 127                        # page 0 stands in for no page: its NaN must not get in
    table[0, 1], table[0, 3], table[1, 0] = -1, 10, 1 << 30
    table[2, :] = -5                             # nothing there at all: zeros
    lens[1] = 10 ** 9                            # cut to the table
    table[table == 0] = -1
    q, q64 = rounded(rng, (3 * new, heads, d), BF16, 0.3)
    got = cache.attend(gpu_pool(pool), 0, gpu_batch((table, lens, cu), new), q.cuda(), causal=False)
    ref = C.attend(pool, 0, (table, lens, cu), q64, page, causal=False)
    check_attend(got, ref, 200, d, BF16)
    assert (got[2 * new:] == 0).all()


def test_attend_tokens_that_see_nothing():
    """A sequence that holds fewer tokens than it has rows: its earliest rows are zeros; so are all of an empty one."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(15)
    page, d, heads, kv = 16, 64, 4, 2
    pool = make_pool(rng, 1, 4, kv, d, page)
    table = np.array([[1, 2], [0, 3]], dtype=np.int32)
    batch = (table, np.array([3, 0], dtype=np.int32), np.array([0, 8, 10], dtype=np.int32))
    q, q64 = rounded(rng, (10, heads, d), BF16)
    for causal in (True, False):
        got = cache.attend(gpu_pool(pool), 0, gpu_batch(batch, 8), q.cuda(), causal=causal)
        check_attend(got, C.attend(pool, 0, batch, q64, page, causal=causal), 3, d, BF16)
        assert (got[8:] == 0).all() and (not causal or (got[:5] == 0).all())


@pytest.mark.parametrize("new", [5, 80])
def test_attend_nan_reaches_only_those_that_see_it(new):
    """A NaN value (or key) of a token is seen by that token and later ones, and by nobody before."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(16)
    page, d, heads, kv, held = 16, 64, 4, 2, 93
    pool = make_pool(rng, 1, 6, kv, d, page)
    batch = make_batch(rng, [(held, new)], page, 6)
    at = held - new + 3                          # the fourth new token
    ko, vo = C.orders(page, d)
    p = batch[0][0, at // page]
    pool["v"][0, p, 0, vo[at % page, 7]] = 127   # kv head 0: channel 7 of its value
    pool["k"][0, p, 1, ko[at % page, 9]] = 255   # kv head 1: its key
    q, q64 = rounded(rng, (new, heads, d), BF16, 0.3)
    got = cache.attend(gpu_pool(pool), 0, gpu_batch(batch, new), q.cuda()).float().cpu().numpy()
    nan = np.isnan(got)
    want = np.zeros_like(nan)
    want[3:, 0:2, 7] = True
    want[3:, 2:4, :] = True
    assert np.array_equal(nan, want)
    clean = {x: y.copy() for x, y in pool.items()}
    for x in "kv":
        clean[x][(clean[x] & 127) == 127] = 0
    o, w, x = C.attend(clean, 0, batch, q64, page)
    check_attend(torch.from_numpy(np.where(nan, o, got)[:3]), (o[:3], w[:3], x[:3]), held, d, BF16)


def test_attend_offsets_past_32_bits():
    """Pages whose bytes lie beyond 4 GB of their array."""
    from paper_2605_15684_amd import cache
    page, d, kv, heads, pages = 64, 128, 8, 8, 67000
    free = torch.cuda.mem_get_info()[0]
    if free < 24 << 30:
        pytest.skip("needs 24 GB")
    g = cache.alloc(1, pages, kv, d, page)
    assert g.k.numel() > 1 << 32
    rng = np.random.default_rng(17)
    ids = [pages - 1, 0, pages - 2, 66000]
    batch = (np.array([ids], dtype=np.int32), np.array([250], dtype=np.int32), np.array([0, 250], dtype=np.int32))
    k, k64 = rounded(rng, (250, kv, d), BF16)
    v, v64 = rounded(rng, (250, kv, d), BF16)
    cache.append(g, 0, gpu_batch(batch, 250), k.cuda(), v.cuda())
    small = make_pool(rng, 1, 4, kv, d, page)
    sbatch = (np.array([[0, 1, 2, 3]], dtype=np.int32),) + batch[1:]
    C.append(small, 0, sbatch, k64, v64, page)
    at = torch.tensor(ids, device="cuda")
    got = {"k": g.k.view(torch.uint8)[:, at].cpu().numpy(), "v": g.v.view(torch.uint8)[:, at].cpu().numpy()}
    order_k, order_v = C.orders(page, d)
    for x, order in (("k", order_k), ("v", order_v)):      # 250 of 256 tokens are written
        assert np.array_equal(got[x][0, :3], small[x][0, :3])
        assert np.array_equal(got[x][0, 3][:, order[:58]], small[x][0, 3][:, order[:58]])
    q, q64 = rounded(rng, (1, heads, d), BF16, 0.3)
    one = (batch[0], batch[1], np.array([0, 1], dtype=np.int32))
    got = cache.attend(g, 0, gpu_batch(one, 1), q.cuda())
    check_attend(got, C.attend(small, 0, (sbatch[0],) + one[1:], q64, page), 250, d, BF16)
    # compaction moves them below
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[at] = 1
    t, r, info = cache.compact(g, table, refs)
    assert info.tolist() == [4, 3] and t.tolist() == [[3, 0, 2, 1]]
    again = cache.attend(g, 0, gpu_batch((t.cpu().numpy(),) + one[1:], 1), q.cuda())
    assert torch.equal(again, got)


# ---- lists -----------------------------------------------------------------------

LISTED = [  # page, D, heads, kv, dtype, causal, keep, sequences
    (16, 64, 4, 2, BF16, True, 3, [(200, 1), (10, 1), (100, 4)]),
    (64, 128, 16, 4, BF16, True, 5, [(1000, 1), (640, 1)]),
    (32, 64, 24, 1, BF16, False, 4, [(300, 20)]),                         # 24 query heads to a kv head
    (16, 128, 3, 3, F32, True, 6, [(150, 3), (20, 20)]),
    (64, 64, 2, 1, F32, True, 2, [(500, 1)]),
    (16, 64, 32, 32, BF16, True, 3, [(150, 130)]),                        # a wave per row
    (32, 128, 64, 32, F32, True, 2, [(140, 131)]),
    (32, 64, 48, 16, BF16, True, 5, [(300, 131), (40, 9)]),               # the same with 3 query heads to a kv head
    (16, 128, 128, 16, BF16, True, 7, [(260, 140)]),                      # 8
    (64, 64, 144, 16, BF16, False, 3, [(400, 133)]),                      # 9
    (64, 128, 16, 4, BF16, True, 40, [(5000, 2), (130, 1)]),              # long lists: parts that are joined
    (16, 64, 6, 2, F32, True, 150, [(3500, 1), (900, 2)]),
    (64, 128, 6, 2, F32, True, 8, [(1000, 1), (640, 3)]),                 # 8 waves to a row
    (32, 64, 3, 3, F32, False, 12, [(700, 2)]),
]


def any_lists(rng, rows, kv, keep, columns):
    """Lists no select would write: any count, any order, pages twice, pages that are none."""
    lists = rng.integers(-2, columns + 2, (rows, kv, 1 + keep)).astype(np.int32)
    lists[..., 0] = rng.integers(-1, keep + 3, (rows, kv))
    return lists


@pytest.mark.parametrize("page,d,heads,kv,dtype,causal,keep,seqs", LISTED)
def test_attend_lists(page, d, heads, kv, dtype, causal, keep, seqs):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(page + d + heads + keep)
    pages, rows = sum(-(-h // page) for h, _ in seqs) + 2, sum(n for _, n in seqs)
    pool = make_pool(rng, 1, pages, kv, d, page)
    batch = make_batch(rng, seqs, page, pages)
    q, q64 = rounded(rng, (rows, heads, d), dtype, 0.3)
    lists = any_lists(rng, rows, kv, keep, batch[0].shape[1])
    lists[0, 0, 0] = 0
    got = cache.attend(gpu_pool(pool), 0, gpu_batch(batch, max(n for _, n in seqs)), q.cuda(), causal=causal,
                       lists=torch.from_numpy(lists).cuda())
    check_attend(got, C.attend(pool, 0, batch, q64, page, lists, causal), keep * page, d, dtype)
    assert (got[0, : heads // kv] == 0).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,kv,group", [(5, 2, 4), (137, 16, 1), (130, 16, 5), (130, 16, 12)])
def test_attend_lists_nan(d, new, kv, group):
    """NaN in every place that no listed token holds; then one key and one value that are seen."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(new + d + group)
    page, held, keep = 16, 403, 9
    clean = make_pool(rng, 1, 30, kv, d, page)
    batch = make_batch(rng, [(held, new)], page, 30)
    table, pages = batch[0][0], -(-held // page)
    lists = np.full((new, kv, 1 + keep), -1, dtype=np.int32)
    for r in range(new):
        own = (held - new + r) // page
        for h in range(kv):
            n = int(rng.integers(1, keep + 1))
            lists[r, h, 0] = n
            lists[r, h, 1:1 + n] = rng.permutation(np.append(rng.permutation(own)[:n - 1], own))
    assert (lists[..., 0] > 0).all() and lists.max() < pages
    ko, vo = C.orders(page, d)
    pool = {x: y.copy() for x, y in clean.items()}
    for x, order in (("k", ko), ("v", vo)):
        kept = np.zeros((30, page * d), dtype=bool)          # the last page: tokens behind the sequence are NaN
        for i in range(pages):
            kept[table[i], order[: min(held - i * page, page)].ravel()] = True
        pool[x][0][np.broadcast_to(~kept[:, None], pool[x][0].shape)] = 127
    q, q64 = rounded(rng, (new, kv * group, d), BF16, 0.3)
    run = lambda: cache.attend(gpu_pool(pool), 0, gpu_batch(batch, new), q.cuda(), lists=torch.from_numpy(lists).cuda())
    ref = C.attend(clean, 0, batch, q64, page, lists, True)
    check_attend(run(), ref, keep * page, d, BF16)
    at = held - new - 3                                      # a token that all rows see whose list has its page
    pool["k"][0, table[at // page], 0, ko[at % page, 9]] = 255
    pool["v"][0, table[at // page], 1, vo[at % page, 7]] = 127
    got = run().float().cpu().numpy().reshape(new, kv, group, d)
    want = np.zeros(got.shape, dtype=bool)
    sees = [[at // page in lists[r, h, 1:1 + lists[r, h, 0]] for h in range(kv)] for r in range(new)]
    for r in range(new):
        want[r, 0] = sees[r][0]
        want[r, 1, :, 7] = sees[r][1]
    assert want.any() and not want.all(axis=(0, 2, 3)).any()
    assert np.array_equal(np.isnan(got), want)


SELECTS = [  # page, D, heads, kv, dtype, causal, keep, first, last, sequences
    (16, 64, 4, 2, BF16, True, 4, 1, 1, [(300, 1), (10, 1), (64, 1), (65, 1)]),
    (64, 128, 16, 4, BF16, True, 6, 1, 1, [(1500, 3), (384, 1), (385, 1), (0, 0)]),
    (16, 128, 6, 1, F32, True, 5, 0, 2, [(400, 90)]),
    (32, 64, 3, 3, BF16, False, 3, 1, 2, [(500, 40), (33, 33)]),          # nothing to choose: first + last = keep
    (16, 64, 2, 1, BF16, True, 9, 2, 3, [(5000, 2)]),                     # more pages than a workgroup takes at once
    (16, 128, 8, 2, F32, True, 300, 1, 1, [(9000, 1)]),
    (16, 64, 2, 2, BF16, True, 50, 1, 1, [(100, 5)]),                     # more places than the table has columns
    (16, 128, 4, 2, BF16, True, 20, 1, 2, [(3000, 40), (9, 9), (100, 17), (5000, 16)]),   # tiles of 16 tokens
    (16, 64, 3, 1, F32, False, 7, 2, 1, [(8000, 33), (640, 8)]),          # the same, half of the LDS
    (32, 128, 2, 1, F32, True, 260, 1, 1, [(30000, 20)]),                 # 938 pages, 258 of them chosen
    (16, 64, 2, 1, BF16, True, 5, 1, 1, [(17000, 1), (40, 1)]),           # too many pages for the LDS
    (16, 128, 2, 1, BF16, True, 11, 1, 1, [(20000, 18), (500, 9)]),       # the same in tiles
    (16, 64, 1, 1, BF16, True, 6, 1, 1, [(18400, 1), (18500, 20)]),       # the last that fit, the first that do not
    (16, 64, 32, 32, BF16, True, 30, 1, 1, [(20000, 40)]),                # many rows: a wave ranks one
    (16, 64, 64, 64, F32, False, 400, 0, 2, [(50000, 17)]),               # the same, longer
    (16, 64, 1, 1, BF16, True, 2000, 1, 1, [(150000, 1)]),                # more pages than registers of a workgroup
    (16, 64, 2, 2, BF16, True, 120, 1, 1, [(2000, 1), (2300, 12), (5000, 9), (9000, 1), (12000, 3)]),   # half of them
    (16, 64, 2, 2, F32, True, 300, 0, 1, [(5000, 1), (6100, 1), (8000, 1), (16000, 1)]),   # negative ones among them
    (16, 64, 2, 1, F32, True, 1800, 1, 1, [(40000, 1), (30000, 3), (18500, 2)]),           # the same, longer
]


@pytest.mark.parametrize("page,d,heads,kv,dtype,causal,keep,first,last,seqs", SELECTS)
def test_select(page, d, heads, kv, dtype, causal, keep, first, last, seqs):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(page + d + heads + keep)
    pages, rows = sum(-(-h // page) for h, _ in seqs) + 2, sum(n for _, n in seqs)
    pool = make_pool(rng, 1, pages, kv, d, page)
    batch = make_batch(rng, seqs, page, pages)
    q, q64 = rounded(rng, (rows, heads, d), dtype)
    lists = torch.full((rows, kv, 1 + keep), -7, dtype=torch.int32, device="cuda")
    cache.select(gpu_pool(pool), 0, gpu_batch(batch, max(n for _, n in seqs)), q.cuda(), keep=keep, first=first,
                 last=last, causal=causal, lists=lists)
    want = C.select(pool, 0, batch, q64, page, keep, first, last, causal)
    assert np.array_equal(lists.cpu().numpy(), want)


@pytest.mark.parametrize("columns", [40, 300, 700, 1152, 1500])
@pytest.mark.parametrize("max_new", [2, 8])
def test_select_ties_nan_and_missing_pages(columns, max_new):
    """Equal scores keep the lower page, zeros of both signs are equal, NaN and missing pages come last; the hint
    and rows of no sequence do not matter."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(18)
    page, d, kv, keep = 16, 64, 2, 8
    pool = make_pool(rng, 1, 40, kv, d, page)
    pool["kmean"][0, 1::3] = pool["kmean"][0, 1]            # a third of the pages alike
    pool["kmean"][0, 2::9] = 0.0
    pool["kmean"][0, 5::9] = -0.0
    pool["kmean"][0, 7, 0, 3] = np.nan
    pool["kmean"][0, 11] = np.inf
    table = np.full((3, columns), -1, dtype=np.int32)        # the width of the table picks the kernel
    table[:, :40] = np.arange(40)
    table[1, 5:20] = -1
    table[1, 21] = 40
    table[2, 3:39] = 77                                      # fewer pages there than places
    lens, cu = np.array([640, 635, 630], dtype=np.int32), np.array([1, 3, 4, 5], dtype=np.int32)
    q, q64 = rounded(rng, (6, 4, d), BF16)
    lists = torch.full((6, kv, 1 + keep), -7, dtype=torch.int32, device="cuda")
    for hint in (None, 20):
        cache.select(gpu_pool(pool), 0, gpu_batch((table, lens, cu), max_new, hint), q.cuda(), keep=keep, lists=lists)
        with np.errstate(invalid="ignore"):
            want = C.select(pool, 0, (table, lens, cu), q64, page, keep)
        assert np.array_equal(lists.cpu().numpy(), want)


# ---- pages -------------------------------------------------------------------------

def _gpu_rows(*arrays):
    return [torch.from_numpy(x.copy()).cuda() for x in arrays]


def _same_rows(gpu, host):
    for a, b in zip(gpu, host):
        assert np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("pages,rows,columns,page", [(7, 1, 1, 16), (60, 5, 9, 16), (3000, 40, 50, 64), (50, 30, 7, 32),
                                                     (20000, 33, 700, 16), (300, 1200, 3, 16)])
def test_pages(pages, rows, columns, page):
    """reserve, fork, release, compact in turn, with what the header allows: rows twice, rows that are none, pools
    that run out of pages."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(pages)
    pool = make_pool(rng, 3 if pages < 5000 else 1, pages, 3 if pages < 5000 else 1, 64, page)
    gpool = gpu_pool(pool)
    table = np.full((rows, columns), -1, dtype=np.int32)
    lens, refs = np.zeros(rows, dtype=np.int32), np.zeros(pages, dtype=np.int32)
    g = _gpu_rows(table, lens, refs)
    for turn in range(6 if pages < 5000 else 2):
        some = rng.random(rows) < 0.6
        lens[some] = rng.integers(0, columns * page + page, int(some.sum()))
        lens[~some] = np.minimum(lens[~some] + 1, columns * page)
        g[1].copy_(torch.from_numpy(lens))
        want = C.reserve(table, lens, refs, page)
        assert tuple(cache.reserve(gpool, *g).tolist()) == want
        _same_rows(g, (table, lens, refs))
        n = int(rng.integers(0, rows + 3))
        gone = rng.integers(-1, rows + 1, n).astype(np.int32)
        want = C.release(table, lens, refs, gone)
        assert tuple(cache.release(gpool, *g, torch.from_numpy(gone).cuda()).tolist()) == want
        _same_rows(g, (table, lens, refs))
        src, dst = rng.integers(-1, rows + 1, (2, n)).astype(np.int32)
        # a dst row that is not empty would lose its pages: empty them first
        C.release(table, lens, refs, dst)
        cache.release(gpool, *g, torch.from_numpy(dst).cuda())
        want = C.fork(pool, table, lens, refs, src, dst, page)
        got = cache.fork(gpool, *g, torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda())
        assert tuple(got.tolist()) == want
        _same_rows(g, (table, lens, refs))
        assert_same_pool(host_pool(gpool), pool)
        table, refs, live, moved = C.compact(pool, table, refs)
        if turn % 2:
            t, r, info = cache.compact(gpool, g[0], g[2])
            g = [t, g[1], r]
        else:                                            # in place
            t, r, info = cache.compact(gpool, g[0], g[2], g[0], g[2])
            assert t is g[0] and r is g[2]
        assert info.tolist() == [live, moved]
        _same_rows(g, (table, lens, refs))
        assert_same_pool(host_pool(gpool), pool)


def test_copy_pages():
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(20)
    a, b = make_pool(rng, 2, 9, 3, 64, 16), make_pool(rng, 2, 5, 3, 64, 16)
    ga, gb = gpu_pool(a), gpu_pool(b)
    src, dst = np.array([8, 0, 9, 3, -1, 4], dtype=np.int32), np.array([1, 4, 0, 5, 2, 3], dtype=np.int32)
    cache.copy_pages(ga, *_gpu_rows(src, dst), to=gb)
    for x, y in ((8, 1), (0, 4), (4, 3)):
        for n in a:
            b[n][:, y] = a[n][:, x]
    assert_same_pool(host_pool(gb), b)
    cache.copy_pages(ga, *_gpu_rows(np.array([1, 2], dtype=np.int32), np.array([7, 5], dtype=np.int32)))
    for x, y in ((1, 7), (2, 5)):
        for n in a:
            a[n][:, y] = a[n][:, x]
    assert_same_pool(host_pool(ga), a)


def test_binding_refusals():
    from paper_2605_15684_amd import cache
    pool = cache.alloc(1, 4, 2, 64, 16)
    table, lens, refs = cache.alloc_rows(pool, 2, 2000)
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    batch = cache.Batch(table, lens, cu, 1)
    k = torch.zeros(2, 2, 64, dtype=BF16, device="cuda")
    q = torch.zeros(2, 4, 64, dtype=BF16, device="cuda")
    lists = torch.zeros(2, 2, 4, dtype=torch.int32, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    bad = [lambda: cache.append(pool, 0, batch, k.cpu(), k), lambda: cache.append(pool, 0, batch, k, k.float()),
           lambda: cache.append(pool, 0, batch, k.half(), k.half()), lambda: cache.append(pool, 0, batch, k[:, :1], k[:, :1]),
           lambda: cache.append(pool, 0, batch, k, torch.zeros(2, 4, 64, dtype=BF16, device="cuda")[:, ::2]),
           lambda: cache.attend(pool, 0, batch, q[..., :32]), lambda: cache.attend(pool, 0, batch, q[0]),
           lambda: cache.attend(pool, 0, batch, torch.zeros(2, 4, 128, dtype=BF16, device="cuda")[..., ::2]),
           lambda: cache.attend(pool, 0, batch, q, out=q.float()), lambda: cache.attend(pool, 0, batch, q, out=q[:1]),
           lambda: cache.attend(pool, 0, batch, q, lists=lists[:1]), lambda: cache.attend(pool, 0, batch, q, lists=lists.long()),
           lambda: cache.attend(pool, 0, batch, q, scratch=q.cpu()), lambda: cache.select(pool, 0, batch, q, keep=3, lists=lists[:, :1]),
           lambda: cache.Batch(table, lens[:1], cu, 1), lambda: cache.Batch(table, lens, cu[:2], 1),
           lambda: cache.Batch(table[:, ::2], lens, cu, 1), lambda: cache.reserve(pool, table, lens, refs[:2]),
           lambda: cache.fork(pool, table, lens, refs, one, cu), lambda: cache.release(pool, table, lens, refs, one.long()),
           lambda: cache.compact(pool, table, refs, table_out=table[:1]), lambda: cache.copy_pages(pool, one, cu),
           lambda: cache.PagedCache(pool.k, pool.v[:, :2], pool.scale, pool.kmean),
           lambda: cache.PagedCache(pool.k, pool.v, pool.scale.double(), pool.kmean)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {i} was not refused")
    for st, call in ((1, lambda: cache.attend(pool, 1, batch, q)), (1, lambda: cache.append(pool, -1, batch, k, k)),
                     (1, lambda: cache.select(pool, 0, batch, q, keep=0)), (1, lambda: cache.select(pool, 0, batch, q, keep=2, first=2)),
                     (2, lambda: cache.attend(pool, 0, batch, q[:, :3])), (1, lambda: cache.attend(pool, 0, batch, q, scale=float("nan"))),
                     (4, lambda: cache.select(pool, 0, batch, q, keep=3, scratch=torch.zeros(4, device="cuda"))),
                     (4, lambda: cache.attend(pool, 0, batch, q, scratch=torch.zeros(4, device="cuda"))),
                     (4, lambda: cache.reserve(pool, table, lens, refs, scratch=torch.zeros(4, device="cuda")))):
        with pytest.raises(cache.SsbaError) as e:
            call()
        assert e.value.status == st
    # nothing to do is no error
    none = torch.zeros(0, 4, 64, dtype=BF16, device="cuda")
    assert cache.attend(pool, 0, batch, none).shape == none.shape
    cache.append(pool, 0, batch, none[:, :2], none[:, :2])
    empty = one[:0]
    assert cache.fork(pool, table, lens, refs, empty, empty).tolist() == [0, 0]
    assert cache.release(pool, table, lens, refs, empty).tolist() == [0, 0]
    cache.copy_pages(pool, empty, empty)


# ---- a run of all of them -------------------------------------------------------------

def test_calls_without_rows():
    """An idle batch: no row in any packed array, nothing written."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(20)
    pool = make_pool(rng, 1, 6, 2, 64, 16)
    g = gpu_pool(pool)
    batch = gpu_batch(make_batch(rng, [(20, 0), (33, 0)], 16, 6), 0)
    k, q = torch.empty(0, 2, 64, dtype=BF16, device="cuda"), torch.empty(0, 8, 64, dtype=BF16, device="cuda")
    cache.append(g, 0, batch, k, k)
    lists = cache.select(g, 0, batch, q, keep=2)
    assert lists.shape == (0, 2, 3)
    assert cache.attend(g, 0, batch, q).shape == q.shape == cache.attend(g, 0, batch, q, lists=lists).shape
    assert_same_pool(host_pool(g), pool)
    # rows of no sequence, among idle ones: left as they are
    batch = gpu_batch(make_batch(rng, [(20, 0), (33, 0)], 16, 6), 1)
    out = torch.full((3, 8, 64), 7.0, dtype=BF16, device="cuda")
    cache.append(g, 0, batch, out[:, :2], out[:, 2:4])
    cache.attend(g, 0, batch, torch.ones_like(out), out=out)
    assert (out == 7).all()
    assert_same_pool(host_pool(g), pool)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_generation(dtype):
    """Prompts, steps, a fork, steps of both branches, a release, compaction, steps: two layers, dense and selected
    attention against the oracle at every step."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(21)
    layers, page, d, heads, kv, keep = 2, 16, 64, 4, 2, 3
    pool = make_pool(rng, layers, 40, kv, d, page)
    gpool = gpu_pool(pool)
    rows, columns = 4, 9
    g = cache.alloc_rows(gpool, rows, columns)
    table, lens, refs = np.full((rows, columns), -1, dtype=np.int32), np.zeros(rows, dtype=np.int32), np.zeros(40, dtype=np.int32)

    def step(new):
        lens[:] += new
        g[1].copy_(torch.from_numpy(lens))
        C.reserve(table, lens, refs, page)
        assert cache.reserve(gpool, *g)[1] == 0
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        batch, gbatch = (table, lens, cu), cache.Batch(g[0], g[1], torch.from_numpy(cu).cuda(), int(max(new)), int(max(lens)))
        for layer in range(layers):
            (k, k64), (v, v64), (q, q64) = (rounded(rng, (int(cu[-1]), n, d), dtype) for n in (kv, kv, heads))
            cache.append(gpool, layer, gbatch, k.cuda(), v.cuda())
            C.append(pool, layer, batch, k64, v64, page)
            o = cache.attend(gpool, layer, gbatch, q.cuda())
            check_attend(o, C.attend(pool, layer, batch, q64, page), 200, d, dtype)
            lists = cache.select(gpool, layer, gbatch, q.cuda(), keep=keep)
            want = C.select(pool, layer, batch, q64, page, keep)
            assert np.array_equal(lists.cpu().numpy(), want)
            o = cache.attend(gpool, layer, gbatch, q.cuda(), lists=lists)
            check_attend(o, C.attend(pool, layer, batch, q64, page, want), 200, d, dtype)
        assert_same_pool(host_pool(gpool), pool)
        _same_rows(g, (table, lens, refs))

    step(np.array([37, 0, 80, 0]))
    for _ in range(3):
        step(np.array([1, 0, 1, 0]))
    src, dst = np.array([0, 2], dtype=np.int32), np.array([1, 3], dtype=np.int32)
    C.fork(pool, table, lens, refs, src, dst, page)
    cache.fork(gpool, *g, *_gpu_rows(src, dst))
    for _ in range(2):
        step(np.array([1, 1, 2, 1]))
    gone = np.array([2], dtype=np.int32)
    C.release(table, lens, refs, gone)
    cache.release(gpool, *g, *_gpu_rows(gone))
    table, refs, live, _ = C.compact(pool, table, refs)
    cache.compact(gpool, g[0], g[2], g[0], g[2])
    assert (refs[live:] == 0).all()
    for _ in range(3):
        step(np.array([1, 1, 0, 5]))


def test_captured_step_replays_with_new_lengths():
    """A whole step (reserve, append, select, attention both ways) in a graph: lengths, tables and inputs change
    between replays, with eager work in between."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(22)
    page, d, heads, kv, keep, seqs = 16, 64, 4, 2, 3, 3
    pool = make_pool(rng, 1, 60, kv, d, page)
    gpool, eager = gpu_pool(pool), gpu_pool(pool)
    state = cache.alloc_rows(gpool, seqs, 20)
    twin = cache.alloc_rows(eager, seqs, 20)
    cu = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    k, v = (torch.zeros(seqs, kv, d, dtype=BF16, device="cuda") for _ in range(2))
    q = torch.zeros(seqs, heads, d, dtype=BF16, device="cuda")

    def step(p, s):
        s[1].add_(1)
        cache.reserve(p, *s)
        b = cache.Batch(s[0], s[1], cu, 1)
        cache.append(p, 0, b, k, v)
        lists = cache.select(p, 0, b, q, keep=keep)
        return cache.attend(p, 0, b, q), lists, cache.attend(p, 0, b, q, lists=lists)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        start = [x.clone() for x in state]
        step(gpool, state)                      # first calls outside the capture
        for x, y in zip(state, start):
            x.copy_(y)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        outs = step(gpool, state)
    for x, y in zip(state, start):
        x.copy_(y)
    for p in (gpool, eager):                    # the first call has put a token into the graph's pool
        for name in ("k", "v"):
            getattr(p, name).view(torch.uint8).copy_(torch.from_numpy(pool[name]))
        p.scale.copy_(torch.from_numpy(pool["scale"]))
        p.kmean.copy_(torch.from_numpy(pool["kmean"]))
    torch.cuda.synchronize()
    for turn in range(70):
        if turn == 20:
            for s in (state, twin):
                s[1][1] = 150                   # one sequence jumps ahead
        for t in (k, v, q):
            t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape))).to(BF16))
        graph.replay()
        want = step(eager, twin)
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), turn
        for a, b in zip(state, twin):
            assert torch.equal(a, b)
    a, b = host_pool(gpool), host_pool(eager)
    assert_same_pool(a, b)


def test_two_streams_and_repeats():
    """The same calls on another stream, and again, give the same bits."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(23)
    page, d, heads, kv = 16, 128, 8, 2
    seqs = [(700, 1), (90, 1), (333, 1)]
    pool = make_pool(rng, 1, 80, kv, d, page)
    g, batch = gpu_pool(pool), gpu_batch(make_batch(rng, seqs, page, 80), 1)
    q = rounded(rng, (3, heads, d), BF16)[0].cuda()
    torch.cuda.synchronize()
    one = cache.attend(g, 0, batch, q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams * 3:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(cache.attend(g, 0, batch, q, lists=cache.select(g, 0, batch, q, keep=6)))
            outs.append(cache.attend(g, 0, batch, q))
    torch.cuda.synchronize()
    assert all(torch.equal(x, one) for x in outs[1::2]) and all(torch.equal(x, outs[0]) for x in outs[::2])
