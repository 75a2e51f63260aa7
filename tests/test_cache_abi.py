"""Host-side checks of the cache's C ABI and binding (no GPU, nothing is
launched): every refusal of include/ssba_cache.h, workspace sizes."""
import ctypes
import os

import pytest
import torch

from paper_2605_15684_amd import _lib

P = 0x10000            # an aligned address that no refused call may touch
OK, ARG, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2605_15684_amd import build
        build.build()
    return _lib.load()


def cache(**kw):
    a = dict(layers=2, pages=10, kv_heads=2, head_dim=64, page=16, k=P, v=P, scale=P, kmean=P)
    return _lib.CacheDesc(**{**a, **kw})


def batch(**kw):
    a = dict(seqs=3, max_pages=8, rows=3, max_new=1, max_len=0, table=P, lens=P, cu=P)
    return _lib.CacheBatch(**{**a, **kw})


def query(**kw):
    a = dict(heads=4, dtype=_lib.DT_BF16, causal=1, keep=4, first=1, last=1, softmax_scale=0.0)
    return _lib.CacheQuery(**{**a, **kw})


def rows(**kw):
    return _lib.CachePages(**{**dict(rows=3, max_pages=8, table=P, lens=P, refs=P), **kw})


BAD_CACHE = [(dict(layers=0), SHAPE), (dict(pages=0), SHAPE), (dict(kv_heads=-1), SHAPE), (dict(head_dim=96), UNSUPPORTED),
             (dict(page=8), UNSUPPORTED), (dict(page=128), UNSUPPORTED), (dict(pages=(1 << 24) + 1), UNSUPPORTED),
             (dict(kv_heads=1025), UNSUPPORTED), (dict(layers=65535), UNSUPPORTED)]
BAD_ARRAYS = [(dict(k=None), ARG), (dict(v=P + 8), ARG), (dict(scale=P + 4), ARG), (dict(kmean=P + 2), ARG)]
BAD_BATCH = [(dict(seqs=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(rows=-1), SHAPE), (dict(max_new=-1), SHAPE),
             (dict(max_len=-1), SHAPE), (dict(seqs=65536), UNSUPPORTED), (dict(max_pages=1 << 27), UNSUPPORTED)]
BAD_BATCH_ARRAYS = [(dict(table=None), ARG), (dict(lens=P + 2), ARG), (dict(cu=None), ARG)]
BAD_QUERY = [(dict(heads=0), SHAPE), (dict(heads=3), SHAPE), (dict(dtype=2), ARG), (dict(causal=2), ARG),
             (dict(softmax_scale=float("nan")), ARG), (dict(softmax_scale=float("inf")), ARG), (dict(keep=-1), ARG),
             (dict(keep=(1 << 24) + 1), UNSUPPORTED), (dict(heads=2 * 65536), UNSUPPORTED)]
BAD_STRIDES = [(dict(q_stride_t=-64, q_stride_h=64), SHAPE), (dict(q_stride_t=260, q_stride_h=64), UNSUPPORTED),
               (dict(q_stride_t=256, q_stride_h=32), SHAPE), (dict(q_stride_t=32, q_stride_h=64), SHAPE)]


def append(lib, c=None, layer=0, b=None, dtype=_lib.DT_BF16, k=P, v=P, st=0, sh=0):
    return lib.ssba_cache_append(c or cache(), layer, b or batch(), dtype, k, v, st, sh, None)


def select(lib, c=None, layer=0, b=None, q=None, query_=P, lists=P, lists_bytes=1 << 40, scratch=P, bytes_=1 << 40):
    return lib.ssba_cache_select(c or cache(), layer, b or batch(), q or query(), query_, lists, lists_bytes, scratch,
                                 bytes_, None)


def attend(lib, c=None, layer=0, b=None, q=None, query_=P, lists=None, lists_bytes=1 << 40, o=P, scratch=P,
           bytes_=1 << 40):
    return lib.ssba_cache_attend(c or cache(), layer, b or batch(), q or query(), query_, lists, lists_bytes, o, scratch,
                                 bytes_, None)


CALLS = [append, select, attend]


@pytest.mark.parametrize("call", CALLS, ids=lambda f: f.__name__)
def test_refusals_shared_by_the_token_calls(lib, call):
    for kw, st in BAD_CACHE + BAD_ARRAYS:
        assert call(lib, c=cache(**kw)) == st, kw
    for kw, st in BAD_BATCH + BAD_BATCH_ARRAYS:
        assert call(lib, b=batch(**kw)) == st, kw
    assert call(lib, layer=-1) == ARG and call(lib, layer=2) == ARG


@pytest.mark.parametrize("call", [select, attend], ids=lambda f: f.__name__)
def test_refusals_of_queries(lib, call):
    for kw, st in BAD_QUERY + BAD_STRIDES:
        assert call(lib, q=query(**kw)) == st, kw
    assert call(lib, query_=None) == ARG and call(lib, query_=P + 8) == ARG
    assert call(lib, q=query(dtype=_lib.DT_F32), query_=P + 2) == ARG


def test_refusals_of_append(lib):
    assert append(lib, k=None) == ARG and append(lib, v=P + 8) == ARG and append(lib, dtype=7) == ARG
    assert append(lib, dtype=_lib.DT_F32, k=P + 2) == ARG
    for st, sh in ((-128, 64), (64, 64 - 8), (32, 64)):
        assert append(lib, st=st, sh=sh) == SHAPE, (st, sh)
    assert append(lib, st=132, sh=64) == UNSUPPORTED
    assert append(lib, c=cache(kv_heads=1024, pages=1 << 24), b=batch(seqs=65535, max_pages=1 << 20, max_new=1 << 20,
                                                                      rows=1 << 20)) == UNSUPPORTED
    # nothing to do: nothing is launched
    assert append(lib, b=batch(rows=0), k=None, v=None) == OK and append(lib, b=batch(max_new=0)) == OK


def test_refusals_of_select(lib):
    for kw in (dict(keep=0), dict(first=-1), dict(last=0), dict(first=3, last=2), dict(first=2 ** 31 - 1)):
        assert select(lib, q=query(**kw)) == ARG, kw
    assert select(lib, lists=None) == ARG and select(lib, lists=P + 2) == ARG
    assert select(lib, lists_bytes=4 * 3 * 2 * 5 - 1) == WORKSPACE
    size = ctypes.c_size_t(0)
    long = batch(max_pages=2048)
    assert lib.ssba_cache_select_workspace_size(cache(), long, query(), size) == OK and size.value == 8 * 3 * 2 * 2048
    assert select(lib, b=long, bytes_=size.value - 1) == WORKSPACE
    assert select(lib, b=long, scratch=None) == ARG and select(lib, b=long, scratch=P + 8) == ARG
    assert lib.ssba_cache_select_workspace_size(cache(), batch(), query(), size) == OK and size.value == 0
    assert select(lib, b=batch(rows=0), lists=None, scratch=None) == OK
    for kw, st in BAD_QUERY + [(dict(keep=0), ARG)]:
        assert lib.ssba_cache_select_workspace_size(cache(), batch(), query(**kw), size) == st, kw


def test_refusals_of_attend(lib):
    assert attend(lib, o=None) == ARG and attend(lib, o=P + 8) == ARG and attend(lib, lists=P + 2) == ARG
    assert attend(lib, q=query(keep=0), lists=P) == ARG
    assert attend(lib, lists=P, lists_bytes=4 * 3 * 2 * 5 - 1) == WORKSPACE
    assert attend(lib, q=query(o_stride_t=256, o_stride_h=60)) == SHAPE
    assert attend(lib, q=query(o_stride_t=260, o_stride_h=64)) == UNSUPPORTED
    size = ctypes.c_size_t(0)
    long = batch(max_pages=4096)
    assert lib.ssba_cache_attend_workspace_size(cache(), long, query(), 0, size) == OK and size.value > 0
    assert attend(lib, b=long, bytes_=size.value - 1) == WORKSPACE
    assert attend(lib, b=long, scratch=None) == ARG and attend(lib, b=long, scratch=P + 4) == ARG
    assert lib.ssba_cache_attend_workspace_size(cache(), long, query(keep=0), 1, size) == ARG
    assert attend(lib, b=batch(rows=0), query_=None, o=None) == OK
    assert attend(lib, b=batch(max_new=0), query_=None, o=None) == OK
    assert attend(lib, b=batch(seqs=65535, rows=1 << 30, max_new=1 << 30)) == UNSUPPORTED


def test_null_descriptors(lib):
    size = ctypes.c_size_t(0)
    c, b, q, r = cache(), batch(), query(), rows()
    assert lib.ssba_cache_append(None, 0, b, 0, P, P, 0, 0, None) == ARG
    assert lib.ssba_cache_append(c, 0, None, 0, P, P, 0, 0, None) == ARG
    for f, tail in ((lib.ssba_cache_select, (P, P, 1 << 40, P, 1 << 40, None)),
                    (lib.ssba_cache_attend, (P, None, 0, P, P, 1 << 40, None))):
        assert f(None, 0, b, q, *tail) == ARG and f(c, 0, None, q, *tail) == ARG and f(c, 0, b, None, *tail) == ARG
    assert lib.ssba_pages_workspace_size(None, r, 1, size) == ARG and lib.ssba_pages_workspace_size(c, None, 1, size) == ARG
    assert lib.ssba_pages_copy(None, c, 1, P, P, None) == ARG and lib.ssba_pages_copy(c, None, 1, P, P, None) == ARG
    assert lib.ssba_cache_select_workspace_size(c, b, q, None) == OK


PAGE_CALLS = {
    "reserve": lambda lib, c, p, n, x, y, info, s, b: lib.ssba_pages_reserve(c, p, info, s, b, None),
    "fork": lambda lib, c, p, n, x, y, info, s, b: lib.ssba_pages_fork(c, p, n, x, y, info, s, b, None),
    "release": lambda lib, c, p, n, x, y, info, s, b: lib.ssba_pages_release(c, p, n, x, info, s, b, None),
    "compact": lambda lib, c, p, n, x, y, info, s, b: lib.ssba_pages_compact(c, p, x, y, info, s, b, None),
}


@pytest.mark.parametrize("name", sorted(PAGE_CALLS))
def test_refusals_of_the_page_calls(lib, name):
    def call(c=None, p=None, n=2, x=P, y=P, info=P, s=P, b=1 << 40):
        return PAGE_CALLS[name](lib, c or cache(), p or rows(), n, x, y, info, s, b)

    for kw, st in BAD_CACHE:
        assert call(c=cache(**kw)) == st, kw
    for kw, st in ((dict(rows=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(rows=1 << 16, max_pages=1 << 15), UNSUPPORTED),
                   (dict(table=None), ARG), (dict(lens=None), ARG), (dict(refs=P + 2), ARG)):
        assert call(p=rows(**kw)) == st, kw
    assert call(info=None) == ARG and call(info=P + 2) == ARG and call(s=None) == ARG and call(s=P + 8) == ARG
    size = ctypes.c_size_t(0)
    n = 2 if name in ("fork", "release") else 0
    assert lib.ssba_pages_workspace_size(cache(), rows(), n, size) == OK
    assert call(b=size.value - 1) == WORKSPACE
    if name in ("fork", "release"):
        assert call(n=-1) == SHAPE and call(x=None) == ARG and call(x=P + 1) == ARG
        assert call(n=(1 << 24) + 1) == UNSUPPORTED
    if name in ("fork", "compact"):
        assert call(y=None) == ARG and call(y=P + 2) == ARG
        for kw, st in BAD_ARRAYS:
            assert call(c=cache(**kw)) == st, kw
    assert lib.ssba_pages_workspace_size(cache(), rows(), -1, size) == SHAPE


def test_refusals_of_copy(lib):
    for kw in (dict(layers=3), dict(kv_heads=1), dict(head_dim=128), dict(page=32)):
        assert lib.ssba_pages_copy(cache(), cache(**kw), 1, P, P, None) == SHAPE, kw
    for kw, st in BAD_CACHE + BAD_ARRAYS:
        assert lib.ssba_pages_copy(cache(**kw), cache(), 1, P, P, None) == st, kw
    assert lib.ssba_pages_copy(cache(), cache(), -1, P, P, None) == SHAPE
    assert lib.ssba_pages_copy(cache(), cache(), 1, None, P, None) == ARG
    assert lib.ssba_pages_copy(cache(), cache(), 1, P, P + 2, None) == ARG
    assert lib.ssba_pages_copy(cache(), cache(), 0, None, None, None) == OK


def test_binding_refuses_host_tensors_and_wrong_types(lib):
    from paper_2605_15684_amd import cache as C
    k = torch.zeros(1, 2, 1, 16 * 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale, kmean = torch.zeros(1, 2, 1, 2), torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16)
    for bad in ((k, k, scale, kmean), (None, k, scale, kmean), (k[0], k, scale, kmean), (k.float(), k, scale, kmean)):
        with pytest.raises(ValueError):
            C.PagedCache(*bad)
    i = torch.zeros(2, dtype=torch.int32)
    for bad in ((None, i, i), (torch.zeros(2, 3, dtype=torch.int32), i, i), (torch.zeros(2, 3), i, i)):
        with pytest.raises(ValueError):
            C.Batch(*bad, 1)


def test_c99_caller(tmp_path, lib):
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("gcc not installed")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    libdir, exe = os.path.dirname(_lib.LIB_PATH), tmp_path / "cache_from_c"
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(root, "include"),
                        os.path.join(root, "tests", "c", "cache_from_c.c"), "-L", libdir, "-lssba",
                        f"-Wl,-rpath,{libdir}", "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
