"""Calls of the cache's binding that it has to refuse, or to answer, on the GPU."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def small(tokens, page=16, d=64, kv=4, columns=4):
    """A pool of 8 pages and a batch of one sequence that brings `tokens` tokens."""
    from paper_2605_15684_amd import cache
    pool = cache.alloc(1, 8, kv, d, page)
    for x in (pool.k, pool.v):
        x.view(torch.uint8).zero_()
    pool.scale.fill_(1.0)
    pool.kmean.zero_()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return pool, cache.Batch(i32([[0, 1, 2, 3][:columns]]), i32([tokens]), i32([0, tokens]), tokens)


@pytest.mark.parametrize("tokens", [1, 3])
def test_broadcast_tensors_are_refused(tokens):
    from paper_2605_15684_amd import cache
    pool, batch = small(tokens)
    k = torch.zeros(tokens, 4, 64, dtype=BF16, device="cuda")
    q = torch.zeros(tokens, 8, 64, dtype=BF16, device="cuda")
    shared = torch.zeros(1, 1, 64, dtype=BF16, device="cuda")
    ks, qs = shared.expand(tokens, 4, 64), shared.expand(tokens, 8, 64)
    for call in (lambda: cache.append(pool, 0, batch, ks, ks), lambda: cache.append(pool, 0, batch, k, ks),
                 lambda: cache.attend(pool, 0, batch, qs), lambda: cache.attend(pool, 0, batch, q, out=qs),
                 lambda: cache.select(pool, 0, batch, qs, keep=2)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("page,d,dtype", [(16, 64, BF16), (64, 128, BF16), (32, 128, F32), (64, 64, F32)])
def test_append_to_pages_with_other_scales(page, d, dtype):
    """Pages that came with scales of any positive value: older tokens keep what they hold, page by page as the oracle
    has it; some pages are completed, some scales reach what is new, some do not."""
    from paper_2605_15684_amd import cache
    from oracle import cache_oracle as C
    from _cache import assert_same_pool, gpu_batch, gpu_pool, host_pool, make_batch, make_pool, rounded
    rng = np.random.default_rng(30)
    kv, scales = 2, [0.75, 3.1, 2.0 ** -70, 1e-40, 2.0 ** -64, 0.5, 1.0000001, 2.0 ** 120, 1.5 * 2.0 ** 100, 1e-3]
    seqs = [(page - 2, 3), (page, 5), (page + 4, 9)] * 10
    need = [-(-h // page) for h, _ in seqs]
    pool = make_pool(rng, 1, sum(need) + 2, kv, d, page)
    table, lens, cu = make_batch(rng, seqs, page, sum(need) + 2)
    for s in range(len(seqs)):
        for which in (0, 1):
            pool["scale"][0, table[s, :need[s]], :, which] = scales[(s // 3 + 3 * which) % len(scales)]
    rows = int(cu[-1])
    size = torch.from_numpy(10.0 ** rng.uniform(-6, 3, (rows, 1, 1)))
    (k, k64), (v, v64) = (rounded(rng, (rows, kv, d), dtype, size) for _ in range(2))
    g = gpu_pool(pool)
    cache.append(g, 0, gpu_batch((table, lens, cu), 9), k.cuda(), v.cuda())
    C.append(pool, 0, (table, lens, cu), k64, v64, page)
    assert_same_pool(host_pool(g), pool)


@pytest.mark.parametrize("new", [1, 9])
def test_rows_of_no_sequence_do_not_matter(new):
    """Rows in front of, behind and between sequences: whatever they hold, results are the same, and they stay."""
    from paper_2605_15684_amd import cache
    from _cache import assert_same_pool, gpu_batch, gpu_pool, host_pool, make_batch, make_pool, rounded
    rng = np.random.default_rng(31)
    page, d, heads, kv = 16, 64, 4, 2
    pool = make_pool(rng, 1, 22, kv, d, page)
    table, lens, cu = make_batch(rng, [(140, new), (90, 0), (100, new)], page, 22)
    cu += 3
    rows = int(cu[-1]) + 2
    inside = torch.zeros(rows, dtype=torch.bool)
    inside[3:int(cu[-1])] = True
    results = []
    for fill in (0.0, float("nan"), float("inf")):
        rng = np.random.default_rng(32)
        (k, _), (v, _), (q, _) = (rounded(rng, (rows, n, d), BF16) for n in (kv, kv, heads))
        for x in (k, v, q):
            x[~inside] = fill
        g, b = gpu_pool(pool), gpu_batch((table, lens, cu), new)
        lists = torch.full((rows, kv, 5), -7, dtype=torch.int32, device="cuda")
        out, listed = (torch.full((rows, heads, d), 5.0, dtype=BF16, device="cuda") for _ in range(2))
        cache.append(g, 0, b, k.cuda(), v.cuda())
        cache.select(g, 0, b, q.cuda(), keep=4, lists=lists)
        cache.attend(g, 0, b, q.cuda(), out=out)
        cache.attend(g, 0, b, q.cuda(), lists=lists, out=listed)
        assert (lists.cpu()[~inside] == -7).all()
        assert (out.cpu()[~inside] == 5).all() and (listed.cpu()[~inside] == 5).all()
        results.append((lists, out, listed, host_pool(g)))
    for other in results[1:]:
        assert all(torch.equal(x, y) for x, y in zip(other[:3], results[0][:3]))
        assert_same_pool(other[3], results[0][3])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("columns", [3, 1200])
def test_sequences_that_outgrow_their_table(columns, dtype):
    """Tokens past the table's last page are not written, and move nothing that is there: the ones that still fit are at
    their own positions, the last pages keep what they held (a sharing row may read it); queries past it see all."""
    from paper_2605_15684_amd import cache
    from oracle import cache_oracle as C
    from _cache import assert_same_pool, gpu_batch, gpu_pool, host_pool, make_pool, rounded
    from test_gpu_cache import check_attend
    rng = np.random.default_rng(33)
    page, d, heads, kv, keep = 16, 64, 4, 2, 2
    end = columns * page
    over = [(end + 1, 1), (end + 5, 10), (end + 70, 10), (2 ** 31 - 1, 3), (end, 4), (end - 3, 2)]
    pool = make_pool(rng, 1, 6 * 3, kv, d, page)
    table = np.full((len(over), columns), -1, dtype=np.int32)
    table[:, -3:] = rng.permutation(18).reshape(6, 3)
    batch = (table, np.array([h for h, _ in over], dtype=np.int32), np.cumsum([0] + [n for _, n in over]).astype(np.int32))
    rows = int(batch[2][-1])
    (k, k64), (v, v64), (q, q64) = (rounded(rng, (rows, n, d), dtype, 0.3) for n in (kv, kv, heads))
    g, b = gpu_pool(pool), gpu_batch(batch, 10)
    cache.append(g, 0, b, k.cuda(), v.cuda())
    before = host_pool(gpu_pool(pool))
    C.append(pool, 0, batch, k64, v64, page)
    assert_same_pool(host_pool(g), pool)
    for s in (0, 2, 3):                              # nothing of these fits
        for x in before:
            assert np.array_equal(before[x][0, table[s, -3:]], pool[x][0, table[s, -3:]])
    lists = cache.select(g, 0, b, q.cuda(), keep=keep)
    want = C.select(pool, 0, batch, q64, page, keep)
    assert np.array_equal(lists.cpu().numpy(), want)
    check_attend(cache.attend(g, 0, b, q.cuda()), C.attend(pool, 0, batch, q64, page), end, d, dtype)
    check_attend(cache.attend(g, 0, b, q.cuda(), lists=lists), C.attend(pool, 0, batch, q64, page, want), end, d, dtype)
