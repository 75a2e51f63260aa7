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
