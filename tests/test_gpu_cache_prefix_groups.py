"""Attention over shared prefixes of many groups without a hint about their sizes: the groups' column tiles are packed.
On the GPU against the fp64 oracle, within the bounds of tests/test_gpu_cache.py."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C

from _cache import gpu_batch, gpu_pool, make_pool, rounded
from test_gpu_cache import check_attend
from test_gpu_cache_shared_parts import make, scratch
from test_gpu_cache_spans import BF16, F32, prefix_of

pytestmark = pytest.mark.gpu


def packed(g, batch, q, new, first, shared, max_seqs, prefix_len):
    """Whether the prefixes' scratch is less than the columns of the largest possible group for each of them."""
    rows, heads, d = q.shape
    grp = heads // g.kv_heads
    columns = -(-grp * min(new * max_seqs, rows) // 16) * 16
    need = scratch(g, batch, q, new, prefix_len, first, shared, max_seqs, prefix_len)     # nothing behind them
    return need < len(shared) * g.kv_heads * columns * (d + 2) * 4


def even(n, pre, members):
    return [(pre + i % 3, members) for i in range(n)]


GROUPS = [  # page, D, heads, kv heads, dtype, causal, groups: (pages of the prefix, [(tokens behind it, new)])
    (16, 64, 2, 1, BF16, True, even(70, 1, [(3, 1)])),
    (16, 64, 8, 2, BF16, True, [(1 + i % 4, [(2 + (i + j) % 9, 1 + (i + j) % 3) for j in range(1 + i % 3)]) for i in range(66)]),
    (64, 128, 16, 4, BF16, True, even(20, 1, [(1, 1), (70, 1), (9, 0)])),
    (32, 64, 8, 2, BF16, True, even(9, 2, [(40, 20), (23, 23), (60, 7)])),                # several tiles a group
    (16, 128, 8, 1, BF16, False, even(10, 3, [(45, 40)])),
    (64, 64, 6, 1, BF16, True, [(2, [(200, 150), (180, 180)])] + even(12, 1, [(5, 2)])),  # one large group
    (16, 64, 6, 2, F32, True, even(30, 2, [(4, 1), (20, 5)])),
    (32, 128, 5, 1, F32, True, [(0, [(7, 3)]), (3, [])] * 6 + even(9, 1, [(33, 9), (1, 1)])),
    (64, 64, 4, 1, BF16, True, even(6, 2, [(2200, 1)]) + even(6, 1, [(5, 2)])),           # and the rests in parts
    (16, 128, 20, 1, F32, True, even(5, 4, [(700, 3), (650, 2)]) + even(5, 1, [(9, 1)])),
]


@pytest.mark.parametrize("page,d,heads,kv,dtype,causal,groups", GROUPS)
def test_many_groups(page, d, heads, kv, dtype, causal, groups):
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(page + d + heads + len(groups))
    pool, batch, first, shared = make(rng, groups, page, kv, d)
    length, new = int(batch[1].max()), int(np.diff(batch[2]).max())
    q, q64 = rounded(rng, (int(batch[2][-1]), heads, d), dtype, 0.2)
    g, dev = gpu_pool(pool), gpu_batch(batch, new, length)
    longest = max(shared) * page
    assert packed(g, batch, q, new, first, shared, len(batch[1]), longest)
    ref = C.attend(pool, 1, C.shared_table(batch, first, shared), q64, page, causal=causal)
    for hints in ((), (None, longest), (max(len(m) for _, m in groups), longest)):
        got = cache.attend_shared(g, 1, dev, prefix_of(first, shared, *hints), q.cuda(), causal=causal)
        check_attend(got, ref, length, d, dtype)


@pytest.mark.parametrize("first,pages", [
    (list(range(13)), [4] * 12), ([0] * 12 + [12], [4] * 12), (list(range(12, -1, -1)), [4] * 12),
    ([0, 5, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12], [4, 3, 2, 1] * 3), ([0, 1, 2, 3, 4, 5, 11, 7, 8, 9, 10, 11, 12], [1, 4, 4] * 4),
    ([-5, -1, 0, 0, 3, 3, 3, 9, 100, 100, 101, 102, 103], [4] * 12), ([2, 2, 3, 4, 5, 6, 7, 8, 9, 9, 9, 10, 11], [100, -1, 4] * 4),
    ([0, 3, 3, 6, 6, 9, 9, 12, 0, 3, 6, 9, 12], [4] * 12), ([2 ** 31 - 1, -2 ** 31] * 6 + [12], [2 ** 31 - 1] * 12)])
def test_whatever_the_groups_say(first, pages):
    """All rows of the table name the same pages, so every grouping means the same; nothing leaves the arrays."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(3)
    page, d, heads, kv = 16, 64, 8, 2
    pool = make_pool(rng, 1, 8, kv, d, page)
    table = np.tile(np.arange(5, dtype=np.int32), (12, 1))
    g = gpu_pool(pool)
    for lens, news in (([70, 66, 80, 65] * 3, [2, 1, 0, 1] * 3), ([70, 20, 33, 1, 80, 64] * 2, [2, 3, 1, 1, 7, 0] * 2),
                       ([3, 0, 70, 10 ** 9] * 3, [5, 2, 1, 1] * 3)):
        batch = (table, np.array(lens, dtype=np.int32), np.concatenate([[0], np.cumsum(news)]).astype(np.int32))
        q, q64 = rounded(rng, (sum(news), heads, d), BF16, 0.3)
        assert packed(g, batch, q, max(news), first, pages, 12, 64)
        got = cache.attend_shared(g, 0, gpu_batch(batch, max(news)), prefix_of(first, pages, None, 64), q.cuda())
        check_attend(got, C.attend(pool, 0, batch, q64, page), 80, d, BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_and_replayed(dtype):
    """Groups, rows and lengths change between replays of one graph; each replay gives what the eager call gives."""
    from paper_2605_15684_amd import cache
    rng = np.random.default_rng(6)
    page, d, heads, kv, seqs = 16, 64, 4, 2, 24
    pool = make_pool(rng, 1, 90, kv, d, page)
    g = gpu_pool(pool)
    table = np.concatenate([np.tile(np.arange(5, dtype=np.int32), (seqs, 1)), 10 + np.arange(seqs * 3, dtype=np.int32).reshape(seqs, 3)], 1)
    lens = 80 + rng.integers(3, 45, seqs).astype(np.int32)
    cu = np.arange(seqs + 1, dtype=np.int32)
    dev = gpu_batch((table, lens, cu), 3)
    pre = prefix_of(list(range(seqs + 1)), [5] * seqs, None, 80)
    q, q64 = rounded(rng, (2 * seqs, heads, d), dtype, 0.3)
    assert packed(g, (table, lens, cu), q, 3, list(range(seqs + 1)), [5] * seqs, seqs, 80)
    dq, out = q.cuda(), torch.full(q.shape, 3.0, dtype=dtype, device="cuda")
    call = lambda o: cache.attend_shared(g, 0, dev, pre, dq, out=o)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    ints = lambda x: torch.tensor(x, dtype=torch.int32)
    one = [1] * seqs
    for first, pages, news, held in ((list(range(seqs + 1)), [5] * seqs, one, lens), ([0] + [seqs] * seqs, [3] * seqs, one, lens),
                                     ([0, 1, 5] + [9] * 10 + [20] * 12, [4] * seqs, [1, 2, 3, 0] * 6, lens),
                                     ([min(2 * i, seqs) for i in range(seqs + 1)], [5, 2] * 12, [0, 3] * 12, lens - 40),
                                     (list(range(seqs + 1)), [5] * seqs, one, lens)):
        at = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        for dst, src in ((pre.first, ints(first)), (pre.pages, ints(pages)), (dev.cu, torch.from_numpy(at)),
                         (dev.lens, torch.from_numpy(held.astype(np.int32)))):
            dst.copy_(src)
        want = torch.full_like(out, 3.0)
        call(want)
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert (out[int(at[-1]):] == 3.0).all(), "rows of no sequence were written"
        check_attend(out[:int(at[-1])], C.attend(pool, 0, (table, held.astype(np.int32), at), q64[:int(at[-1])], page), 128, d, dtype)
