"""Attention over shared prefixes where what is behind the prefix is in parts of its own, so that a launch of its own
joins both, on the GPU against the fp64 oracle, within the bounds of tests/test_gpu_cache.py."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache_oracle as C

from _cache import gpu_batch, gpu_pool, make_pool, rounded
from test_gpu_cache import check_attend
from test_gpu_cache_spans import BF16, F32, prefix_of, shared_batch

pytestmark = pytest.mark.gpu


def scratch(pool, batch, q, max_new, max_len, first, shared, max_seqs, prefix_len):
    """Bytes of the scratch of a call with these hints."""
    from paper_2605_15684_amd import _lib, cache
    size = ctypes.c_size_t(0)
    rows, heads, d = q.shape
    b = gpu_batch(batch, max_new, max_len).desc(rows)
    desc = _lib.CacheQuery(heads, cache._DTYPES[q.dtype], 1, 0, 0, 0, 0.0, 0, 0, 0, 0)
    x = _lib.CachePrefix(len(shared), max_seqs, prefix_len, 16, 16)
    _lib.check(_lib.load().ssba_cache_attend_shared_workspace_size(pool.desc, b, desc, x, size), "size")
    return size.value


PARTS = [  # page, D, heads, kv heads, dtype, causal, groups: (pages of the prefix, [(tokens behind it, new)])
    (64, 64, 4, 1, BF16, True, [(5, [(2100, 1), (2500, 1), (7, 1)])]),                                 # 16 columns a workgroup
    (64, 128, 8, 2, BF16, True, [(3, [(2300, 1)]), (0, [(2200, 1)]), (9, [(1, 1), (2111, 0), (600, 2)])]),
    (16, 64, 3, 1, F32, True, [(20, [(2101, 3), (33, 5)]), (4, [(2100, 1)])]),
    (32, 128, 4, 2, F32, True, [(11, [(2200, 1), (2090, 2)])]),
    (16, 64, 6, 1, F32, True, [(40, [(700, 7), (650, 4), (600, 3)]), (3, [(513, 5)])]),                # two tiles, fp32
    (64, 128, 5, 1, F32, False, [(2, [(900, 9), (70, 6)])]),
    (32, 64, 8, 1, BF16, True, [(7, [(2200, 3), (2300, 4)]), (1, [(2150, 2)])]),                       # two tiles
    (64, 128, 8, 1, BF16, True, [(4, [(2100, 7), (1500, 5)])]),                                        # four
    (16, 64, 6, 1, BF16, True, [(30, [(2500, 20), (3000, 17)])]),                                      # eight
    (64, 128, 6, 2, BF16, False, [(6, [(2500, 60), (2000, 41)]), (2, [(1800, 33)])]),                  # sixteen
    (64, 64, 5, 1, BF16, True, [(3, [(2600, 50), (30, 30), (2500, 52)])]),
]


def make(rng, groups, page, kv, d):
    pages, batch, first, shared = shared_batch(rng, groups, page)
    pool = make_pool(rng, 2, pages, kv, d, page)
    orders = C.orders(page, d)
    used = np.zeros(pages, dtype=bool)
    for s, held in enumerate(batch[1]):
        ids = batch[0][s][: -(-int(held) // page)]
        used[ids] = True
        if held % page:
            for which, x in enumerate("kv"):
                pool[x][1, ids[-1]][:, orders[which][held % page:].ravel()] = 127
    for x in "kv":
        pool[x][1, ~used] = 255
    pool["scale"][1, ~used] = np.nan
    # the others' entries of shared pages are not read
    table = batch[0].copy()
    for g, n in enumerate(shared):
        table[first[g] + 1:first[g + 1], :n] = -1
    return pool, (table,) + tuple(batch[1:]), first, shared


@pytest.mark.parametrize("page,d,heads,kv,dtype,causal,groups", PARTS)
def test_rests_in_parts(page, d, heads, kv, dtype, causal, groups):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(page + d + heads)
    pool, batch, first, shared = make(rng, groups, page, kv, d)
    length, new = int(batch[1].max()), int(np.diff(batch[2]).max())
    most, longest = max(len(m) for _, m in groups), max(shared) * page
    q, q64 = rounded(rng, (int(batch[2][-1]), heads, d), dtype, 0.2)
    g, dev = gpu_pool(pool), gpu_batch(batch, new, length)
    short = scratch(g, batch, q, new, longest, first, shared, most, longest)      # nothing behind the prefix
    assert scratch(g, batch, q, new, length, first, shared, most, longest) > short, "the rests are not in parts"
    ref = C.attend(pool, 1, C.shared_table(batch, first, shared), q64, page, causal=causal)
    for hints in ((most, longest), (most, 1), (len(batch[1]), longest), ()):
        got = cache.attend_shared(g, 1, dev, prefix_of(first, shared, *hints), q.cuda(), causal=causal)
        check_attend(got, ref, length, d, dtype)
    # a group of more sequences than max_seqs says is attended by sequence, from its own entries
    full = C.shared_table(batch, first, shared)
    got = cache.attend_shared(g, 1, gpu_batch(full, new, length), prefix_of(first, shared, 1, longest), q.cuda(), causal=causal)
    check_attend(got, ref, length, d, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sequences_of_no_group(dtype):
    """The first and the last sequence are in no group; rows of no sequence keep what they held."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(21)
    page, d, heads, kv = 32, 64, 4, 2
    groups = [(3, [(2200, 1)]), (5, [(2300, 2), (40, 1), (2100, 3)]), (0, [(2250, 1)])]
    pages, batch, first, shared = shared_batch(rng, groups, page)
    pool = make_pool(rng, 1, pages, kv, d, page)
    table, lens, cu = batch
    cu = (cu + 2).astype(np.int32)
    rows = int(cu[-1]) + 3
    batch = (table, lens, cu)
    q, q64 = rounded(rng, (rows, heads, d), dtype, 0.3)
    out = torch.full((rows, heads, d), 5.0, dtype=dtype, device="cuda")
    length = int(lens.max())
    g = gpu_pool(pool)
    assert scratch(g, batch, q, 3, length, first[1:3], shared[1:2], 3, 160) > scratch(g, batch, q, 3, 160, first[1:3], shared[1:2], 3, 160)
    cache.attend_shared(g, 0, gpu_batch(batch, 3, length), prefix_of(first[1:3], shared[1:2], 3, 160), q.cuda(), out=out)
    check_attend(out, C.attend(pool, 0, batch, q64, page), length, d, dtype)
    assert (out[:2] == 5.0).all() and (out[int(cu[-1]):] == 5.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("columns,heads", [(1, 4), (9, 4), (3, 40)])
def test_scales_far_apart(dtype, columns, heads):
    """The prefix's values are 2^80 larger than the rest's and its keys count for nothing, and the other way round."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(9)
    page, d, kv = 16, 64, 2
    for loud in (0, 1):
        pages, batch, first, shared = shared_batch(rng, [(6, [(2117, 1)] * columns)], page)
        pool = make_pool(rng, 1, pages, kv, d, page)
        pre = batch[0][0, :6]
        rest = np.setdiff1d(np.arange(pages), pre)
        big, small = (pre, rest) if loud == 0 else (rest, pre)
        pool["scale"][0, big, :, 1] = 2.0 ** 40
        pool["scale"][0, small, :, 1] = 2.0 ** -40
        pool["scale"][0, big, :, 0] = 2.0 ** -20
        q, q64 = rounded(rng, (columns, heads, d), dtype, 0.3)
        g = gpu_pool(pool)
        assert scratch(g, batch, q, 1, 2213, first, shared, columns, 96) > scratch(g, batch, q, 1, 96, first, shared, columns, 96)
        got = cache.attend_shared(g, 0, gpu_batch(batch, 1, 2213), prefix_of(first, shared, columns, 96), q.cuda())
        check_attend(got, C.attend(pool, 0, batch, q64, page), 2213, d, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_nan_reaches_those_that_see_it(dtype):
    """One in the prefix reaches all sequences of the group, one behind it only its own."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(5)
    page, d, heads, kv = 16, 64, 4, 2
    groups = [(4, [(2100, 1), (2150, 2)]), (2, [(2120, 1)])]
    pages, batch, first, shared = shared_batch(rng, groups, page)
    table, lens, cu = batch
    vo = C.orders(page, d)[1]
    q, _ = rounded(rng, (4, heads, d), dtype, 0.3)
    for where, rows in (((0, 3), [0, 1, 2]), ((0, 70), [0]), ((1, 100), [1, 2]), ((2, 1), [3])):
        pool = make_pool(rng, 1, pages, kv, d, page)
        pool["v"][0, table[where], 1, vo[3, 7]] = 127
        got = cache.attend_shared(gpu_pool(pool), 0, gpu_batch(batch, 2, int(lens.max())), prefix_of(first, shared, 2, 64),
                                  q.cuda())
        want = np.zeros((4, heads, d), dtype=bool)
        want[rows, 2:, 7] = True
        assert np.array_equal(np.isnan(got.float().cpu().numpy()), want), where


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_and_replayed(dtype):
    """Lengths and groups change between replays of one graph; each replay gives what the eager call gives."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(6)
    page, d, heads, kv = 16, 64, 4, 2
    pages, batch, first, shared = shared_batch(rng, [(6, [(2400, 1), (2300, 1)]), (3, [(2200, 1)])], page)
    pool = make_pool(rng, 1, pages, kv, d, page)
    g = gpu_pool(pool)
    length = int(batch[1].max())
    dev = gpu_batch(batch, 1, length)
    pre = prefix_of(first, shared, 2, 96)
    q = rounded(rng, (3, heads, d), dtype, 0.3)[0].cuda()
    q64 = q.double().cpu().numpy()
    out = torch.zeros_like(q)
    call = lambda o: cache.attend_shared(g, 0, dev, pre, q, out=o)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    lens = batch[1]
    for held, groups, n in ((lens, first, shared), (lens - 200, first, [2, 1]), (lens - 2000, [0, 1, 1], [5, 4]),
                            (np.minimum(lens, 70), first, shared), (lens, first, shared)):
        held = held.astype(np.int32)
        dev.lens.copy_(torch.from_numpy(held))
        pre.first.copy_(torch.tensor(groups, dtype=torch.int32))
        pre.pages.copy_(torch.tensor(n, dtype=torch.int32))
        want = torch.zeros_like(q)
        call(want)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        check_attend(out, C.attend(pool, 0, (batch[0], held, batch[2]), q64, page), length, d, dtype)
