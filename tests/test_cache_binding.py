"""What the cache's binding refuses before it calls the library (no GPU: tensors that say they are on one, and nothing
is launched)."""
import importlib
import os
from types import SimpleNamespace

import pytest
import torch

from paper_2605_15684_amd import _lib

POOL = SimpleNamespace(index=0, head_dim=64, kv_heads=4)


@pytest.fixture(scope="module", autouse=True)
def built():
    global cache
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2605_15684_amd import build
        build.build()
    cache = importlib.import_module("paper_2605_15684_amd.cache")


class OnGpu(torch.Tensor):
    """A host tensor that says it is on GPU 0."""
    is_cuda = True

    def get_device(self):
        return 0


def gpu(t):
    return t.as_subclass(OnGpu)


def packed(t, heads=None):
    return cache._packed(gpu(t), None, heads, POOL, None, "x")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_share_memory_are_refused(dtype):
    """Strides (0, 0) mean a contiguous array to the library: a broadcast tensor must not get there with them."""
    x = torch.zeros(6, 4, 64, dtype=dtype)
    one = x[:1, :1]
    for bad in (one.expand(1, 4, 64), one.expand(6, 4, 64), one.expand(6, 1, 64), x[:, :1].expand(6, 4, 64),
                x[:1].expand(6, 4, 64), x.view(-1).as_strided((6, 4, 64), (32, 64, 1)),
                x.view(-1).as_strided((6, 4, 64), (256, 32, 1))):
        with pytest.raises(ValueError, match="must not overlap"):
            packed(bad)


def test_strides_of_what_is_accepted():
    x = torch.zeros(6, 4, 64)
    assert packed(x) == (256, 64)
    assert packed(x[:1]) == (256, 64)
    assert packed(x[:, :1]) == (256, 64)
    assert packed(x[:1, :1]) == (64, 64)
    assert packed(torch.zeros(4, 6, 64).transpose(0, 1)) == (64, 384)          # heads first
    assert packed(torch.zeros(6, 12, 64)[:, 4:8]) == (768, 64)                  # a slice of a projection
    assert packed(x[:0]) == (256, 64) and packed(x[:1].expand(0, 4, 64))[1] == 64


def calls():
    """A pool and a batch of one token that say they are on GPU 0, and its queries."""
    codes = gpu(torch.zeros(2, 4, 4, 16 * 64, dtype=torch.uint8).view(torch.float8_e4m3fn))
    pool = cache.PagedCache(codes, codes, gpu(torch.ones(2, 4, 4, 2)), gpu(torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16)))
    i32 = lambda *x: gpu(torch.tensor(x, dtype=torch.int32))
    return pool, cache.Batch(i32(0, 1).view(1, 2), i32(1), i32(0, 1), 1), gpu(torch.zeros(1, 8, 64))


@pytest.mark.parametrize("scale", [0.0, -0.0, -0.125, 1e-60, float("-inf")])
def test_scales_that_the_library_takes_for_none(scale):
    """Its default, 1 / sqrt(D), stands for every scale <= 0 there: here only None does."""
    pool, batch, q = calls()
    with pytest.raises(ValueError, match="scale"):
        cache.attend(pool, 0, batch, q, scale=scale)


@pytest.mark.parametrize("big", [1 << 32, (1 << 32) + 1, -(1 << 32), 1 << 31, -(1 << 31) - 1])
def test_numbers_that_int32_does_not_hold(big):
    """The library's numbers are int32; ctypes cuts larger ones to their low bits without a word (2^32 is layer 0)."""
    pool, batch, q = calls()
    k = q[:, :4]
    table, lens, cu = batch.table, batch.lens, batch.cu
    for call in (lambda: cache.append(pool, big, batch, k, k), lambda: cache.attend(pool, big, batch, q),
                 lambda: cache.select(pool, big, batch, q, keep=2), lambda: cache.select(pool, 0, batch, q, keep=2, first=big),
                 lambda: cache.select(pool, 0, batch, q, keep=2, first=0, last=big),
                 lambda: cache.Batch(table, lens, cu, big), lambda: cache.Batch(table, lens, cu, 1, big)):
        with pytest.raises(ValueError, match="int32"):
            call()


def wide(rows, columns):
    """A tensor of a shape that no memory has to hold."""
    return gpu(torch.zeros(1, dtype=torch.int32).expand(rows, columns))


def test_shapes_that_int32_does_not_hold(monkeypatch):
    pool, batch, q = calls()
    refs = gpu(torch.zeros(4, dtype=torch.int32))
    monkeypatch.setattr(OnGpu, "is_contiguous", lambda self: True, raising=False)
    table = wide(1, (1 << 32) + 1)
    numbers = wide(1, (1 << 32) + 1)[0]
    for call in (lambda: cache.Batch(table, batch.lens, batch.cu, 1), lambda: cache.reserve(pool, table, batch.lens, refs),
                 lambda: cache.compact(pool, table, refs),
                 lambda: cache.release(pool, batch.table, batch.lens, refs, numbers),
                 lambda: cache.copy_pages(pool, numbers, numbers)):
        with pytest.raises(ValueError, match="int32"):
            call()
