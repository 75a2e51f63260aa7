"""The cache oracle where a sequence is longer than its table."""
import numpy as np

from oracle import cache_oracle as C

from _cache import make_pool


def test_tokens_past_the_table_change_nothing():
    rng = np.random.default_rng(7)
    page, d, kv = 16, 64, 1
    pool = make_pool(rng, 1, 4, kv, d, page)
    pool["scale"][:] = 2.0 ** -4                    # 28: no new token raises it
    x = rng.standard_normal((8, kv, d))
    table = np.array([[2, 0]], dtype=np.int32)
    before = {n: y.copy() for n, y in pool.items()}
    for held, n in ((33, 1), (40, 8), (10 ** 6, 8)):
        C.append(pool, 0, (table, [held], [0, n]), x[:n], x[:n], page)
        assert all(np.array_equal(pool[n_], before[n_]) for n_ in pool)
    C.append(pool, 0, (table, [35], [0, 8]), x, x, page)          # tokens 27 to 31 fit
    ko, vo = C.orders(page, d)
    for name, order in (("k", ko), ("v", vo)):
        got, was = pool[name][0, 0, 0], before[name][0, 0, 0]
        assert np.array_equal(got[order[:11]], was[order[:11]])
        assert np.array_equal(got[order[11:]], C.e4m3(x[:5, 0] * 2.0 ** 4))
    assert np.array_equal(pool["k"][0, 2], before["k"][0, 2])
    q = rng.standard_normal((8, 1, d))
    o, _, _ = C.attend(pool, 0, (table, [35], [0, 8]), q, page)
    for i in range(8):                              # token 27 + i sees 28 + i keys, 32 at most
        one, _, _ = C.attend(pool, 0, (table, [min(28 + i, 32)], [0, 1]), q[i:i + 1], page)
        assert np.array_equal(one[0], o[i])
