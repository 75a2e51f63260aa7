"""Attention over the cache of a window and the first tokens, and of groups that share a prefix, on the GPU against the
fp64 oracle (oracle/cache_oracle.py), within the bounds of tests/test_gpu_cache.py."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C

from _cache import gpu_batch, gpu_pool, make_batch, make_pool, rounded
from test_gpu_cache import check_attend

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

WINDOWS = [  # page, D, heads, kv heads, dtype, causal, window, sinks, sequences
    (64, 64, 1, 1, BF16, True, 1, 0, [(1, 1)]),
    (64, 64, 4, 1, BF16, True, 100, 4, [(4096, 1)]),
    (64, 128, 16, 4, BF16, True, 300, 70, [(1, 1), (64, 1), (65, 1), (1000, 1), (333, 0), (370, 1)]),
    (16, 128, 6, 2, BF16, True, 33, 1, [(17, 1), (16, 1), (15, 1), (500, 1)]),
    (32, 64, 40, 2, BF16, True, 31, 0, [(100, 1), (31, 1)]),
    (16, 64, 6, 2, BF16, True, 7, 3, [(40, 9), (9, 9), (200, 3)]),                 # two column tiles a wave
    (64, 128, 16, 4, BF16, True, 129, 16, [(1000, 8), (300, 5), (2, 2)]),
    (16, 64, 16, 4, BF16, False, 3000, 20, [(5000, 7)]),                           # in parts
    (32, 128, 8, 2, BF16, False, 5, 2, [(300, 12), (12, 12), (77, 1)]),            # four
    (64, 128, 4, 2, BF16, True, 20, 5, [(200, 130), (70, 70), (300, 64)]),         # by columns: windows shorter than a tile
    (64, 128, 4, 2, BF16, True, 150, 0, [(400, 130), (70, 70), (300, 64)]),
    (16, 64, 12, 4, BF16, True, 1000, 17, [(3000, 20), (40, 17), (333, 5)]),       # 64 columns, keys split
    (64, 64, 6, 1, BF16, True, 64, 64, [(1500, 90), (600, 600)]),                  # tiles of 256 columns
    (64, 64, 6, 1, BF16, True, 2147483647, 0, [(1500, 90), (60, 60)]),             # everything
    (64, 64, 6, 1, BF16, True, 1, 2147483647, [(700, 90), (60, 1)]),
    (64, 128, 5, 1, F32, True, 100, 4, [(1, 1), (700, 1)]),
    (16, 64, 6, 2, F32, False, 600, 33, [(1500, 4), (3, 3), (0, 0)]),
    (16, 64, 6, 2, F32, True, 1, 0, [(50, 7), (7, 7), (129, 2)]),
    (32, 128, 4, 2, F32, True, 40, 3, [(150, 60), (64, 33)]),
]


@pytest.mark.parametrize("page,d,heads,kv,dtype,causal,window,sinks,seqs", WINDOWS)
def test_window(page, d, heads, kv, dtype, causal, window, sinks, seqs):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(page + d + heads + len(seqs))
    pages, rows = sum(-(-h // page) for h, _ in seqs) + 3, sum(n for _, n in seqs)
    pool = make_pool(rng, 2, pages, kv, d, page)
    batch = make_batch(rng, seqs, page, pages)
    # what no token sees is NaN, and pages that hold nothing else are not there
    orders = C.orders(page, d)
    for s, (held, n) in enumerate(seqs):
        seen = np.zeros(batch[0].shape[1] * page, dtype=bool)
        for p in range(held - n, held):
            seen[max(p - window + 1, 0):p + 1 if causal else held] = True
            seen[:min(sinks, p + 1 if causal else held)] = True
        for lp in range(-(-held // page)):
            mine = seen[lp * page:(lp + 1) * page]
            if not mine.any():
                batch[0][s, lp] = -1 - lp
                continue
            for which, x in enumerate("kv"):
                pool[x][1, batch[0][s, lp]][:, orders[which][~mine].ravel()] = 127
    q, q64 = rounded(rng, (rows, heads, d), dtype, 0.2)
    ref = C.attend_window(pool, 1, batch, q64, page, window, sinks, causal=causal)
    for hint in (max(h for h, _ in seqs), 1, None):
        got = cache.attend_window(gpu_pool(pool), 1, gpu_batch(batch, max(n for _, n in seqs), hint), q.cuda(),
                                  window=window, sinks=sinks, causal=causal)
        check_attend(got, ref, max(h for h, _ in seqs), d, dtype)


def test_window_over_everything_is_attend():
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(1)
    page, d, heads, kv, seqs = 16, 64, 8, 2, [(100, 3), (77, 1)]
    pool = make_pool(rng, 1, 20, kv, d, page)
    g, batch = gpu_pool(pool), gpu_batch(make_batch(rng, seqs, page, 20), 3, 100)
    q, _ = rounded(rng, (4, heads, d), BF16)
    want = cache.attend(g, 0, batch, q.cuda())
    assert torch.equal(cache.attend_window(g, 0, batch, q.cuda(), window=100), want)


@pytest.mark.parametrize("new", [1, 5, 80])
@pytest.mark.parametrize("what", ["value", "key", "inf"])
def test_window_nan_reaches_only_those_that_see_it(new, what):
    """A NaN of a token is seen by the tokens of the window behind it, a sink's by all."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(16)
    page, d, heads, kv, held, window, sinks = 16, 64, 4, 2, 131, 30, 3
    ko, vo = C.orders(page, d)
    q, q64 = rounded(rng, (new, heads, d), BF16, 0.3)
    for at in (1, sinks, held - new - window + 1, held - new, held - 1 - window, held - window, held - 1):
        if not 0 <= at < held:
            continue
        pool = make_pool(rng, 1, 12, kv, d, page)
        table, lens, cu = batch = make_batch(rng, [(held, new)], page, 12)
        p = table[0, at // page]
        if what == "inf":            # a value far larger than the others, as scales allow: nothing of it elsewhere
            pool["scale"][0, p, :, 1] = 2.0 ** 40
        elif what == "value":
            pool["v"][0, p, 0, vo[at % page, 7]] = 127
        else:
            pool["k"][0, p, 0, ko[at % page, 9]] = 255
        got = cache.attend_window(gpu_pool(pool), 0, gpu_batch(batch, new, held), q.cuda(), window=window, sinks=sinks)
        if what == "inf":
            # More than 16 columns: weights p * vs of less than 2^-22 of the largest are held in steps of 2^-32 of it
            # (the header says so), so a token that sees the page, with a largest weight of at most 2^40, may be off
            # by half a step of each of its keys times the largest code.  The others know nothing of the page.
            o, w, x = C.attend_window(pool, 0, batch, q64, page, window, sinks)
            pos = held - new + np.arange(new)
            lo, hi = at // page * page, at // page * page + page - 1
            sees = (pos >= lo) & ((lo < sinks) | (hi > pos - window))
            coarse = held * 2.0 ** -33 * 2.0 ** 40 * 448 if new * heads // kv > 16 else 0.0
            check_attend(got, (o, w + np.where(sees, coarse * 2.0 ** 8, 0.0)[:, None, None], x), held, d, BF16)
            continue
        want = np.zeros((new, heads, d), dtype=bool)
        for t in range(new):
            pos = held - new + t
            if at <= pos and (at < sinks or at > pos - window):
                want[t, 0:2] = True if what == "key" else np.arange(d) == 7
        assert np.array_equal(np.isnan(got.float().cpu().numpy()), want), at


def test_window_tokens_that_see_nothing_and_long_sequences():
    """Fewer tokens than rows: the earliest see nothing.  A sequence that has outgrown its table: its window counts on."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(15)
    page, d, heads, kv = 16, 64, 4, 2
    pool = make_pool(rng, 1, 5, kv, d, page)
    table = np.array([[1, 2], [0, 3], [4, 2], [1, 0]], dtype=np.int32)
    batch = (table, np.array([3, 0, 40, 2 ** 31 - 1], dtype=np.int32), np.array([0, 8, 10, 15, 16], dtype=np.int32))
    q, q64 = rounded(rng, (16, heads, d), BF16)
    for causal in (True, False):
        for window, sinks in ((12, 2), (1, 0), (6, 0), (2 ** 31 - 1, 0)):
            got = cache.attend_window(gpu_pool(pool), 0, gpu_batch(batch, 8), q.cuda(), window=window, sinks=sinks,
                                      causal=causal)
            # every key of the last sequence's table is behind its window of 2^30 at most
            ref = C.attend_window(pool, 0, batch, q64, page, min(window, 1 << 30), sinks, causal=causal)
            check_attend(got, ref, 32, d, BF16)


def test_window_over_a_ring_of_pages():
    """A table that names the same pages again and again: a stream goes on in them with the window's results."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(6)
    page, d, heads, kv, window, sinks, steps = 16, 64, 4, 1, 40, 5, 300
    ring = 1 + (window + page - 1) // page + 1       # a page of sinks, and those that a window can touch
    most = -(-steps // page)
    table = np.array([[0] + [1 + (i - 1) % ring for i in range(1, most)]], dtype=np.int32)
    whole = np.arange(most, dtype=np.int32)[None]
    small, large = cache.alloc(1, 1 + ring, kv, d, page), cache.alloc(1, most, kv, d, page)
    k, v = (rounded(rng, (steps, kv, d), BF16)[0].cuda() for _ in range(2))
    q = rounded(rng, (steps, heads, d), BF16)[0].cuda()
    at = 0
    for n in [1, 30, 1, 7, 16, 1, 33, 40, 1, 1, 20] * 3:
        n = min(n, steps - at)
        if not n:
            break
        outs = []
        for pool, t in ((small, table), (large, whole)):
            b = gpu_batch((t, np.array([at + n], dtype=np.int32), np.array([0, n], dtype=np.int32)), n)
            if pool is small and n > page:           # a chunk's window must still be there when it attends
                for x in range(0, n, 8):
                    m = min(8, n - x)
                    c = gpu_batch((t, np.array([at + x + m], dtype=np.int32), np.array([0, m], dtype=np.int32)), m)
                    cache.append(pool, 0, c, k[at + x:at + x + m], v[at + x:at + x + m])
                    outs.append(cache.attend_window(pool, 0, c, q[at + x:at + x + m], window=window, sinks=sinks))
                outs = [torch.cat(outs)]
                continue
            cache.append(pool, 0, b, k[at:at + n], v[at:at + n])
            outs.append(cache.attend_window(pool, 0, b, q[at:at + n], window=window, sinks=sinks))
        # the two are split differently: half a step of the output each way, and of the probabilities
        a, b = (x.double() for x in outs)
        assert ((a - b).abs() <= 2 ** -7 * b.abs() + 2 ** -7 * 3).all()
        at += n
    assert at == steps


# ---- shared prefixes ----------------------------------------------------------------

def shared_batch(rng, groups, page, spare=2):
    """groups: [(pages of the prefix, [(tokens behind it, new)])] -> pool pages, batch, first, pages."""
    first, shared, seqs = [0], [], []
    for pre, members in groups:
        first.append(first[-1] + len(members))
        shared.append(pre)
        seqs += [(pre * page + rest, n, pre) for rest, n in members]
    need = sum(shared) + sum(-(-h // page) - p for h, _, p in seqs)
    order = list(rng.permutation(need + 3).astype(np.int32))
    table = np.full((len(seqs), max(-(-h // page) for h, _, _ in seqs) + spare), -1, dtype=np.int32)
    for g, (pre, _) in enumerate(groups):
        ids = [order.pop() for _ in range(pre)]
        for s in range(first[g], first[g + 1]):
            table[s, :pre] = ids
            for lp in range(pre, -(-seqs[s][0] // page)):
                table[s, lp] = order.pop()
    lens = np.array([h for h, _, _ in seqs], dtype=np.int32)
    cu = np.concatenate([[0], np.cumsum([n for _, n, _ in seqs])]).astype(np.int32)
    return need + 3, (table, lens, cu), first, shared


def prefix_of(first, pages, *hints):
    from paper_2605_15684_amd import cache
    return cache.Prefix(torch.tensor(first, dtype=torch.int32, device="cuda"),
                        torch.tensor(pages, dtype=torch.int32, device="cuda"), *hints)


SHARED = [  # page, D, heads, kv heads, dtype, causal, groups
    (64, 64, 1, 1, BF16, True, [(1, [(1, 1)])]),
    (64, 128, 16, 4, BF16, True, [(20, [(1 + 37 * i % 200, 1) for i in range(9)])]),
    (16, 64, 6, 2, BF16, True, [(3, [(5, 1), (20, 0), (1, 1)]), (0, [(33, 2)]), (40, [(16, 1), (2, 2), (17, 1), (100, 3)])]),
    (32, 128, 8, 2, BF16, False, [(9, [(70, 12), (12, 12), (33, 1)]), (2, [(40, 40)])]),
    (16, 64, 12, 4, BF16, True, [(30, [(20, 20), (17, 17), (33, 5)])]),
    (64, 64, 6, 1, BF16, True, [(5, [(90, 90), (100, 100), (1, 1)])]),       # tiles of 256 columns
    (64, 128, 40, 2, BF16, True, [(3, [(1, 1), (64, 1)]), (7, [(65, 1)] * 5)]),
    (16, 128, 5, 1, F32, True, [(7, [(1, 1), (30, 4)]), (1, [(20, 1)])]),
    (16, 64, 24, 8, F32, True, [(60, [(4 + i, 4) for i in range(4)]), (61, [(9, 3)] * 3)]),
    (64, 64, 4, 4, F32, False, [(2, [(50, 50), (3, 3)])]),
    (64, 64, 4, 1, BF16, True, [(1, [(1, 1)] * 130)]),                       # a group of more than 64 sequences
    (16, 64, 2, 1, BF16, True, [(1, [(1, 1)])] * 70),                        # more than 64 groups
]


@pytest.mark.parametrize("page,d,heads,kv,dtype,causal,groups", SHARED)
def test_shared(page, d, heads, kv, dtype, causal, groups):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(page + d + heads + len(groups))
    pages, batch, first, shared = shared_batch(rng, groups, page)
    pool = make_pool(rng, 2, pages, kv, d, page)
    lens, cu = batch[1:]
    length, new = int(lens.max()), int(np.diff(cu).max())
    orders = C.orders(page, d)
    used = np.zeros(pages, dtype=bool)
    for s, held in enumerate(lens):
        ids = batch[0][s][: -(-int(held) // page)]
        used[ids] = True
        if held % page:
            for which, x in enumerate("kv"):
                pool[x][1, ids[-1]][:, orders[which][held % page:].ravel()] = 127
    for x in "kv":
        pool[x][1, ~used] = 255
    pool["scale"][1, ~used] = np.nan
    q, q64 = rounded(rng, (int(cu[-1]), heads, d), dtype, 0.2)
    ref = C.attend(pool, 1, batch, q64, page, causal=causal)
    # the others' entries of shared pages are not read
    table = batch[0].copy()
    for g, n in enumerate(shared):
        table[first[g] + 1:first[g + 1], :n] = -1
    most = max(len(m) for _, m in groups)
    for hints in ((most, max(shared) * page), (most, 0), (), (len(lens), 10 ** 6)):
        got = cache.attend_shared(gpu_pool(pool), 1, gpu_batch((table, lens, cu), new, length),
                                  prefix_of(first, shared, *hints), q.cuda(), causal=causal)
        check_attend(got, ref, length, d, dtype)
    # a group of more sequences than max_seqs says is attended by sequence, from its own entries
    got = cache.attend_shared(gpu_pool(pool), 1, gpu_batch(batch, new, length), prefix_of(first, shared, 1), q.cuda(),
                              causal=causal)
    check_attend(got, ref, length, d, dtype)


@pytest.mark.parametrize("first,pages", [
    ([0, 4], [4]), ([0, 4], [3]), ([0, 4], [100]), ([0, 4], [-3]), ([1, 3], [4]), ([2, 9], [4]), ([0, 0, 4, 4], [4, 4, 4]),
    ([3, 0], [4]), ([0, 3, 1, 4], [4, 2, 4]), ([-5, 2, 2, 100], [4, 1, 3]), ([4, 4], [4]), ([-1, -1], [1]),
    ([2 ** 31 - 1, -2 ** 31], [2 ** 31 - 1])])
def test_shared_whatever_the_groups_say(first, pages):
    """All rows of the table name the same pages, so every grouping means the same; nothing leaves the arrays."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(3)
    page, d, heads, kv = 16, 64, 4, 2
    pool = make_pool(rng, 1, 8, kv, d, page)
    table = np.tile(np.arange(5, dtype=np.int32), (4, 1))
    for lens, news in (([70, 66, 80, 65], [2, 1, 0, 1]), ([70, 20, 33, 1], [2, 3, 1, 1]), ([3, 0, 70, 10 ** 9], [5, 2, 1, 1])):
        batch = (table, np.array(lens, dtype=np.int32), np.concatenate([[0], np.cumsum(news)]).astype(np.int32))
        q, q64 = rounded(rng, (sum(news), heads, d), BF16, 0.3)
        got = cache.attend_shared(gpu_pool(pool), 0, gpu_batch(batch, max(news)), prefix_of(first, pages, 4), q.cuda())
        check_attend(got, C.attend(pool, 0, batch, q64, page), 80, d, BF16)


def test_shared_rows_left_alone_strides_and_scale():
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(12)
    page, d, heads, kv = 32, 64, 6, 3
    for dtype in (BF16, F32):
        pages, (table, lens, cu), first, shared = shared_batch(rng, [(2, [(7, 2), (40, 3)])], page)
        pool = make_pool(rng, 1, pages, kv, d, page)
        cu = cu + 2
        rows = int(cu[-1]) + 3
        qkv, qkv64 = rounded(rng, (rows, 12, d), dtype, 0.3)
        out = torch.full((rows, 8, d), 5.0, dtype=dtype, device="cuda")
        got = cache.attend_shared(gpu_pool(pool), 0, gpu_batch((table, lens, cu), 3), prefix_of(first, shared),
                                  qkv.cuda()[:, 3:9], scale=0.37, out=out[:, 1:7])
        check_attend(got, C.attend(pool, 0, (table, lens, cu), qkv64[:, 3:9], page, scale=0.37), 110, d, dtype)
        rest = out.clone()
        rest[2:int(cu[-1]), 1:7] = 5.0
        assert (rest == 5.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("columns", [1, 30])
def test_shared_scales_far_apart(dtype, columns):
    """The prefix's values are 2^80 larger than the rest's and its keys count for nothing, and the other way round."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(9)
    page, d, heads, kv = 16, 64, 4, 2
    for loud in (0, 1):
        pages, batch, first, shared = shared_batch(rng, [(6, [(17, 1)] * columns)], page)
        pool = make_pool(rng, 1, pages, kv, d, page)
        pre = batch[0][0, :6]
        rest = np.setdiff1d(np.arange(pages), pre)
        big, small = (pre, rest) if loud == 0 else (rest, pre)
        pool["scale"][0, big, :, 1] = 2.0 ** 40
        pool["scale"][0, small, :, 1] = 2.0 ** -40
        pool["scale"][0, big, :, 0] = 2.0 ** -20
        q, q64 = rounded(rng, (columns, heads, d), dtype, 0.3)
        got = cache.attend_shared(gpu_pool(pool), 0, gpu_batch(batch, 1), prefix_of(first, shared), q.cuda())
        check_attend(got, C.attend(pool, 0, batch, q64, page), 113, d, dtype)


def test_fork_and_attend_shared():
    """One prompt, forked: its samples share its complete pages, and attend_shared gives what attend gives."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(2)
    page, d, heads, kv, prompt, samples = 16, 64, 8, 2, 85, 6
    pool = cache.alloc(1, 40, kv, d, page)
    table, lens, refs = cache.alloc_rows(pool, samples, 8)
    lens[0] = prompt
    cache.reserve(pool, table, lens, refs)
    data = lambda n, h: rounded(rng, (n, h, d), BF16)[0].cuda()
    cu = torch.tensor([0] + [prompt] * samples, dtype=torch.int32, device="cuda")
    cache.append(pool, 0, cache.Batch(table, lens, cu, prompt), data(prompt, kv), data(prompt, kv))
    ids = torch.arange(1, samples, dtype=torch.int32, device="cuda")
    cache.fork(pool, table, lens, refs, torch.zeros_like(ids), ids)
    lens += 1
    cache.reserve(pool, table, lens, refs)
    batch = cache.Batch(table, lens, torch.arange(samples + 1, dtype=torch.int32, device="cuda"), 1)
    cache.append(pool, 0, batch, data(samples, kv), data(samples, kv))
    q = data(samples, heads)
    want = cache.attend(pool, 0, batch, q).double()
    prefix = prefix_of([0, samples], [prompt // page], samples)
    got = cache.attend_shared(pool, 0, batch, prefix, q).double()
    # each within half a step of the result and of the probabilities (|v| < 6)
    assert ((got - want).abs() <= 2 ** -7 * want.abs() + 2 ** -7 * 6).all()
