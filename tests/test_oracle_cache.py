"""The cache oracle (oracle/cache_oracle.py) against independent statements of
the same things: torch's e4m3 conversion, full softmax, sorting."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C

from _cache import make_batch, make_pool


def test_e4m3_matches_torch():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, C.E4M3, equal_nan=True)
    finite = np.sort(codes[np.isfinite(codes)])
    mid = (finite[1:] + finite[:-1]) / 2
    x = np.concatenate([finite, mid, np.nextafter(mid, 1e9), np.nextafter(mid, -1e9), [0.0, -0.0],
                        np.random.default_rng(0).standard_normal(4000) * 60])
    x = x[np.abs(x) <= 448].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(C.e4m3(x), want)
    assert C.E4M3[C.e4m3([1e9, -np.inf])].tolist() == [448.0, -448.0] and np.isnan(C.E4M3[C.e4m3([np.nan])]).all()


def test_bf16_matches_torch():
    x = np.random.default_rng(1).standard_normal(5000).astype(np.float32)
    assert np.array_equal(C.to_bf16(x), torch.from_numpy(x).to(torch.bfloat16).float().numpy())


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_byte_orders_are_permutations(page, d):
    for order in C.orders(page, d):
        assert np.array_equal(np.sort(order.ravel()), np.arange(page * d))


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0001, 1), (1.75, -8), (1.76, -7), (0.0, -64), (3.4e38, 120)])
def test_exponent(amax, e):
    assert C.exponent(amax) == e


def test_append_in_pieces_equals_append_at_once_while_no_scale_grows():
    rng = np.random.default_rng(2)
    page, d, kv, n = 16, 64, 2, 39
    k, v = rng.standard_normal((2, n, kv, d))
    k[:, :, 0] = v[:, :, 0] = 3.0         # every token has the page's largest exponent
    k, v = np.clip(k, -3, 3), np.clip(v, -3, 3)
    one = make_pool(rng, 1, 4, kv, d, page)
    two = {x: y.copy() for x, y in one.items()}
    table = np.array([[2, 0, 3]], dtype=np.int32)
    C.append(one, 0, (table, [n], [0, n]), k, v, page)
    at = 0
    for step in (1, 1, 13, 20, 4):
        C.append(two, 0, (table, [at + step], [0, step]), k[at:at + step], v[at:at + step], page)
        at += step
    for x in one:
        assert np.array_equal(one[x], two[x])
    # what is held is within half a step of what was put in
    held = np.concatenate([C.rows_of(one, 0, p, 1, 0, page, d) for p in (2, 0, 3)])[:n]
    assert (np.abs(held - k[:, 1]) <= 2.0 ** -4 * np.abs(k[:, 1]) + 2.0 ** -17).all()


def test_attend_is_softmax_attention():
    rng = np.random.default_rng(3)
    page, d, kv, heads = 16, 64, 2, 6
    pool = make_pool(rng, 1, 9, kv, d, page)
    batch = make_batch(rng, [(37, 5), (70, 1)], page, 9)
    q = rng.standard_normal((6, heads, d))
    o, _, _ = C.attend(pool, 0, batch, q, page)
    for s, (lo, held, n) in enumerate([(0, 37, 5), (5, 70, 1)]):
        ids = batch[0][s][: -(-held // page)]
        for head in range(heads):
            k, v = (torch.from_numpy(np.concatenate([C.rows_of(pool, 0, p, head // 3, w, page, d) for p in ids])[:held])
                    for w in (0, 1))
            mask = torch.ones(n, held, dtype=torch.bool).tril(held - n)
            want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[lo:lo + n, head])[None], k[None],
                                                                    v[None], attn_mask=mask)[0]
            assert np.abs(want.numpy() - o[lo:lo + n, head]).max() < 1e-12
    # lists that name every page change nothing
    lists = np.full((6, kv, 6), -1, dtype=np.int32)
    lists[..., 0] = 5
    lists[..., 1:] = np.arange(5)
    assert np.array_equal(C.attend(pool, 0, batch, q, page, lists)[0], o)


def test_select_ranks_by_score():
    rng = np.random.default_rng(4)
    page, d, kv = 16, 64, 1
    pool = make_pool(rng, 1, 12, kv, d, page)
    batch = make_batch(rng, [(12 * 16 - 3, 1)], page, 12)
    q = rng.standard_normal((1, 2, d))
    scores = pool["kmean"][0, batch[0][0, :12], 0].astype(float) @ q[0].sum(0)
    got = C.select(pool, 0, batch, q, page, keep=5)[0, 0]
    best = 1 + np.argsort(-scores[1:11])[:3]
    assert got.tolist() == [5] + sorted([0, 11] + best.tolist())


def test_pages_of_a_forked_row_and_of_a_compacted_pool():
    rng = np.random.default_rng(5)
    pool = make_pool(rng, 2, 8, 1, 64, 16)
    table = np.full((3, 4), -1, dtype=np.int32)
    lens, refs = np.array([40, 16, 0], dtype=np.int32), np.zeros(8, dtype=np.int32)
    assert C.reserve(table, lens, refs, 16) == (4, 0)
    assert table[0].tolist() == [0, 1, 2, -1] and table[1].tolist() == [3, -1, -1, -1]
    assert C.fork(pool, table, lens, refs, [0], [2], 16) == (1, 0)
    assert table[2].tolist() == [0, 1, 4, -1] and refs.tolist() == [2, 2, 1, 1, 1, 0, 0, 0]
    assert np.array_equal(pool["k"][:, 4], pool["k"][:, 2])
    assert C.release(table, lens, refs, [0, 0, 9]) == (3, 1)
    assert refs.tolist() == [1, 1, 0, 1, 1, 0, 0, 0]
    before = pool["v"][:, 4].copy()
    t, r, live, moved = C.compact(pool, table, refs)
    assert (live, moved) == (4, 1) and r.tolist() == [1, 1, 1, 1, 0, 0, 0, 0] and t[2].tolist() == [0, 1, 2, -1]
    assert np.array_equal(pool["v"][:, 2], before)
