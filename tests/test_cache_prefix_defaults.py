"""cache.Prefix without hints (no GPU: the size calls and plans alone): the scratch of attend_shared goes by the rows of
the call, not by the groups times them, and no hint decides whether a call is accepted."""
import ctypes
import importlib
import itertools
import os

import pytest
import torch

from paper_2605_15684_amd import _lib

OK = 0
P = 0x10000            # an address that is aligned; nothing reads it


@pytest.fixture(scope="module", autouse=True)
def built():
    global L, cache
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2605_15684_amd import build
        build.build()
    L = _lib.load()
    cache = importlib.import_module("paper_2605_15684_amd.cache")


class OnGpu(torch.Tensor):
    """A host tensor that says it is on GPU 0."""
    is_cuda = True

    def get_device(self):
        return 0


def size(groups, each, new, held, prefix_pages, heads=32, kv=8, d=128, page=64, dtype=0, seqs=None, rows=None, **hints):
    """(status, scratch bytes) of groups of `each` sequences with `new` tokens each, as cache.attend_shared asks."""
    seqs = seqs or groups * each
    ints = lambda *n: torch.zeros(*n, dtype=torch.int32).as_subclass(OnGpu)
    x = cache.Prefix(ints(groups + 1), ints(groups), **hints)
    pages = -(-held // page)
    c = _lib.CacheDesc(1, 1 << 20, kv, d, page, P, P, P, P)
    b = _lib.CacheBatch(seqs, pages, seqs * new if rows is None else rows, new, 0, P, P, P)
    q = _lib.CacheQuery(heads, dtype, 1, 0, 0, 0, 0.0, 0, 0, 0, 0)
    out = ctypes.c_size_t(0)
    st = L.ssba_cache_attend_shared_workspace_size(c, b, q, x.desc(seqs), out)
    return st, out.value


SHAPES = list(itertools.product((1, 2, 5, 32, 64, 300), (1, 3, 4, 16), (1, 4, 64, 512), (8192,), (16, 100), (0, 1)))


def test_scratch_without_max_seqs():
    """At most three times what the groups' real size needs."""
    for groups, each, new, held, pre, dtype in SHAPES:
        if groups * each * new > 1 << 16:
            continue
        st, exact = size(groups, each, new, held, pre, dtype=dtype, max_seqs=each, max_len=pre * 64)
        st2, default = size(groups, each, new, held, pre, dtype=dtype, max_len=pre * 64)
        assert st == OK and st2 == OK, (groups, each, new, dtype, st, st2)
        assert default <= 3 * exact, (groups, each, new, dtype, default, exact)


def test_ordinary_sizes_fit():
    """64 prompts of 4 samples, 64 new tokens each, 32 heads on 8, D 128 (once 16 GiB); 32 of 4 with 512 (once refused)."""
    st, need = size(64, 4, 64, 8192, 16)
    assert st == OK and need < 1 << 30
    st, need = size(32, 4, 512, 8192, 16)
    assert st == OK and need < 4 << 30


def test_one_large_group_among_small_ones():
    """max_seqs is that of the large group: the small ones do not each take as much room (13 tiles of 256 columns)."""
    st, need = size(200, 1, 8, 8192, 16, seqs=300, max_seqs=101, max_len=1024)
    assert st == OK and need < 200 * 13 * 256 * 8 * (128 + 2) * 4 // 4


@pytest.mark.parametrize("seqs,held,heads,kv", [(8, 12288, 16, 4), (4, 18432, 16, 4), (2, 100000, 8, 1), (1, 5000, 4, 4)])
def test_rests_are_planned_without_a_hint(seqs, held, heads, kv):
    """A prefix of unknown length is not taken to be all that a sequence holds: what is behind it is in parts, which a
    hint of the whole length leaves out (the prefixes' own parts are the same)."""
    for groups in (1, seqs):
        for dtype in (0, 1):
            kw = dict(each=seqs // groups, new=1, held=held, prefix_pages=0, heads=heads, kv=kv, dtype=dtype)
            whole = -(-held // 64) * 64
            unknown, zero, all_of_it = (size(groups, **kw, **hint) for hint in ({}, dict(max_len=0), dict(max_len=whole)))
            assert unknown == zero and unknown[0] == all_of_it[0] == OK
            assert unknown[1] > all_of_it[1]
