"""The cache oracle's append into pages whose scales are not powers of two: what they hold keeps its value."""
import numpy as np
import pytest

from oracle import cache_oracle as C

from _cache import make_pool


@pytest.mark.parametrize("s,e", [(1.0, 0), (0.75, 0), (1.0000001, 1), (3.1, 2), (2.0 ** -64, -64), (2.0 ** -70, -64),
                                 (1e-40, -64), (2.0 ** 120, 120)])
def test_reach(s, e):
    assert C.reach(s) == e


@pytest.mark.parametrize("scale", [0.75, 3.1, 0.0123, 2.0 ** -5])
def test_older_tokens_keep_their_values(scale):
    """Within half a step of e4m3 (2^-4 of a value, 2^-10 of the new scale) and the fp32 roundings in front of it."""
    rng = np.random.default_rng(6)
    page, d, old = 16, 64, 5
    pool = make_pool(rng, 1, 2, 1, d, page)
    pool["scale"][:] = scale
    before = [C.rows_of(pool, 0, 1, 0, w, page, d)[:old] for w in (0, 1)]
    new = rng.standard_normal((page - old, 1, d)) * 1e-3
    table = np.array([[1]], dtype=np.int32)
    C.append(pool, 0, (table, [page], [0, page - old]), new, new, page)
    for w in (0, 1):
        got, top = C.rows_of(pool, 0, 1, 0, w, page, d), float(pool["scale"][0, 1, 0, w])
        assert top == 2.0 ** C.reach(scale)
        err = np.abs(got[:old] - before[w])
        assert (err <= 2.0 ** -4 * np.abs(before[w]) * (1 + 2.0 ** -20) + 2.0 ** -10 * top).all()
        assert scale != top or not err.any()
    mean = C.rows_of(pool, 0, 1, 0, 0, page, d).mean(0)
    assert (np.abs(pool["kmean"][0, 1, 0] - mean) <= 2.0 ** -8 * np.abs(mean)).all()
