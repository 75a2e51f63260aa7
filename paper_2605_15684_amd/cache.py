"""Torch-facing binding of the paged 8-bit key/value cache (include/ssba_cache.h).

Argument marshalling only, like ssba.py: tensors are checked, outputs and
scratch allocated with torch, and raw device pointers plus the current HIP
stream of the tensors' device passed to the HIP kernels in libssba.so.
Importing fails if the library is not built.

    pool = cache.alloc(layers, pages, kv_heads, head_dim, page=64)
    rows = cache.alloc_rows(pool, rows, max_pages)          # table, lens, refs
    ...                                                     # lens += new tokens
    cache.reserve(pool, *rows)
    batch = cache.Batch(table, lens, cu, max_new)
    cache.append(pool, layer, batch, k, v)                  # [tokens, kv_heads, D]
    o = cache.attend(pool, layer, batch, q)                 # [tokens, heads, D]
    lists = cache.select(pool, layer, batch, q, keep=32)    # or: the best 32 pages of each token
    o = cache.attend(pool, layer, batch, q, lists=lists)
    o = cache.attend_window(pool, layer, batch, q, window=1024, sinks=4)     # or: the last 1024 tokens and the first 4
    prefix = cache.Prefix(first, pages)                     # or, of sequences that share their first pages: reading
    o = cache.attend_shared(pool, layer, batch, prefix, q)  # these once
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import _lib

_L = _lib.load()   # fail loudly at import if the HIP library is missing

__all__ = ["PagedCache", "Batch", "Prefix", "alloc", "alloc_rows", "append", "select", "attend", "attend_window",
           "attend_shared", "reserve", "fork", "release", "compact", "copy_pages", "SsbaError"]

SsbaError = _lib.SsbaError
E4M3 = torch.float8_e4m3fn
_DTYPES = {torch.bfloat16: _lib.DT_BF16, torch.float32: _lib.DT_F32}


# The current HIP stream of a device as a number.  A call of this module costs
# a few microseconds on the host, of which torch.cuda.current_stream() (it
# makes a Stream object) would be two.  Likewise the current device, a quarter
# of a microsecond through torch.cuda.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _call(pool, fn, name: str, *args) -> None:
    """fn(*args, stream) on the current stream of the cache's device."""
    index = pool.index
    if _current_device() == index:
        st = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            st = fn(*args, _raw_stream(index))
    if st:
        _lib.check(st, name)


def _check(t, shape, dtype, index, what: str) -> None:
    """A contiguous tensor of `dtype` on GPU `index`, of `shape` where given."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == index and t.is_contiguous() and \
            (shape is None or t.shape == shape):
        return
    if isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() != index:
        raise ValueError(f"{what}: all tensors must be on one device")
    raise ValueError(f"{what}: expected a contiguous {dtype} GPU tensor" +
                     (f" of shape {tuple(shape)}" if shape is not None else ""))


def _int32(what: str, *numbers) -> None:
    """The library's numbers are int32, and ctypes would cut larger ones."""
    for x in numbers:
        if not -0x80000000 <= x < 0x80000000:
            raise ValueError(f"{what}: outside int32")


def _gpu_of(t, dims: int, what: str) -> int:
    """The GPU of a tensor of `dims` dimensions."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != dims:
        raise ValueError(f"{what}: expected a GPU tensor of {dims} dimensions")
    return t.get_device()


class PagedCache:
    """The arrays of a cache: k, v [layers, pages, kv_heads, page * D] e4m3, scale fp32
    [layers, pages, kv_heads, 2], kmean bf16 [layers, pages, kv_heads, D] (byte order of the pages:
    include/ssba_cache.h).  Holds references to the tensors, copies nothing."""

    __slots__ = ("k", "v", "scale", "kmean", "device", "index", "layers", "pages", "kv_heads", "head_dim", "page", "desc")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, scale: torch.Tensor, kmean: torch.Tensor):
        index = _gpu_of(k, 4, "k")
        _gpu_of(kmean, 4, "kmean")
        shape = k.shape
        layers, pages, kv_heads, size = shape
        d = kmean.shape[3]
        _check(k, None, E4M3, index, "k")
        _check(v, shape, E4M3, index, "v")
        _check(scale, (layers, pages, kv_heads, 2), torch.float32, index, "scale")
        _check(kmean, (layers, pages, kv_heads, d), torch.bfloat16, index, "kmean")
        if d < 1 or size % d:
            raise ValueError("k: the last dimension must be page * D")
        page = size // d
        self.k, self.v, self.scale, self.kmean, self.device, self.index = k, v, scale, kmean, k.device, index
        self.layers, self.pages, self.kv_heads, self.head_dim, self.page = layers, pages, kv_heads, d, page
        self.desc = _lib.CacheDesc(layers, pages, kv_heads, d, page, k.data_ptr(), v.data_ptr(), scale.data_ptr(),
                                   kmean.data_ptr())


class Batch:
    """Sequences of a call: table int32 [seqs, max_pages], lens int32 [seqs] (tokens held, the new ones
    included), cu int32 [seqs + 1] (the new tokens' rows in the packed arrays).  max_new: at least the new
    tokens of any sequence; max_len: about the longest sequence (work is split by it; results are not)."""

    __slots__ = ("table", "lens", "cu", "index", "_desc")

    def __init__(self, table: torch.Tensor, lens: torch.Tensor, cu: torch.Tensor, max_new: int,
                 max_len: Optional[int] = None):
        index = _gpu_of(table, 2, "table")
        seqs, max_pages = table.shape
        max_new, max_len = int(max_new), int(max_len or 0)
        _int32("table, max_new or max_len", seqs, max_pages, max_new, max_len)
        _check(table, None, torch.int32, index, "table")
        _check(lens, (seqs,), torch.int32, index, "lens")
        _check(cu, (seqs + 1,), torch.int32, index, "cu")
        self.table, self.lens, self.cu, self.index = table, lens, cu, index
        self._desc = (seqs, max_pages, max_new, max_len, table.data_ptr(), lens.data_ptr(), cu.data_ptr())

    def desc(self, rows: int) -> _lib.CacheBatch:
        seqs, max_pages, new, length, table, lens, cu = self._desc
        return _lib.CacheBatch(seqs, max_pages, rows, new, length, table, lens, cu)


class Prefix:
    """Groups of consecutive sequences that share their first pages: sequences first[g] .. first[g+1]-1 share pages[g]
    complete pages (first int32 [groups + 1], pages int32 [groups]), named by the table for the first of them.
    max_seqs: at least the sequences of any group (None: those of the batch, which costs time from some tens of groups
    on); max_len: about the longest prefix in tokens (None or 0: unknown; work is split by it, results differ by the
    rounding of partial sums)."""

    __slots__ = ("first", "pages", "index", "max_seqs", "_desc")

    def __init__(self, first: torch.Tensor, pages: torch.Tensor, max_seqs: Optional[int] = None,
                 max_len: Optional[int] = None):
        index = _gpu_of(first, 1, "first")
        _check(first, None, torch.int32, index, "first")
        groups = first.shape[0] - 1
        if groups < 1:
            raise ValueError("first: expected [groups + 1]")
        _check(pages, (groups,), torch.int32, index, "pages")
        max_len = int(max_len or 0)
        max_seqs = None if max_seqs is None else int(max_seqs)
        _int32("first, max_seqs or max_len", groups, max_seqs or 0, max_len)
        if max_seqs is not None and max_seqs < 1 or max_len < 0:
            raise ValueError("max_seqs must be 1 or more, max_len 0 or more")
        self.first, self.pages, self.index, self.max_seqs = first, pages, index, max_seqs
        self._desc = (groups, max_len, first.data_ptr(), pages.data_ptr())

    def desc(self, seqs: int) -> _lib.CachePrefix:
        groups, max_len, first, pages = self._desc
        return _lib.CachePrefix(groups, self.max_seqs or seqs, max_len, first, pages)


def alloc(layers: int, pages: int, kv_heads: int, head_dim: int, page: int = 64, device="cuda") -> PagedCache:
    """A new cache (its contents are arbitrary until appended to)."""
    shape = (layers, pages, kv_heads)
    return PagedCache(torch.empty(shape + (page * head_dim,), dtype=E4M3, device=device),
                      torch.empty(shape + (page * head_dim,), dtype=E4M3, device=device),
                      torch.empty(shape + (2,), dtype=torch.float32, device=device),
                      torch.empty(shape + (head_dim,), dtype=torch.bfloat16, device=device))


def alloc_rows(pool: PagedCache, rows: int, max_pages: int) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Empty page table, lens and refs of `rows` sequences over the pages of `pool`."""
    return (torch.full((rows, max_pages), -1, dtype=torch.int32, device=pool.device),
            torch.zeros(rows, dtype=torch.int32, device=pool.device),
            torch.zeros(pool.pages, dtype=torch.int32, device=pool.device))


def _packed(t, rows, heads, pool: PagedCache, dtype, what: str):
    """Checks a packed [rows, heads, D] tensor (rows, heads, dtype None: any); its (token, head) strides."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 3 and t.dtype in _DTYPES):
        raise ValueError(f"{what}: expected a [tokens, heads, D] GPU tensor, bf16 or fp32")
    if t.get_device() != pool.index:
        raise ValueError(f"{what}: all tensors must be on one device")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype}")
    n, h, d = t.shape
    if d != pool.head_dim or (heads is not None and h != heads) or (rows is not None and n != rows):
        raise ValueError(f"{what}: expected shape [{'tokens' if rows is None else rows}, "
                         f"{'heads' if heads is None else heads}, {pool.head_dim}]")
    st, sh, sc = t.stride()
    if sc != 1 and n * h:
        raise ValueError(f"{what}: channel stride must be 1")
    # Broadcast tensors among them: strides of (0, 0) mean a contiguous array to the library.
    if (n > 1 and h and st < d) or (h > 1 and n and sh < d):
        raise ValueError(f"{what}: rows and heads must not overlap")
    # A dimension of one has no stride that matters; torch may report any.
    if h < 2:
        sh = d
    if n < 2:
        st = h * sh
    return st, sh


def _same_device(pool: PagedCache, batch: Batch) -> None:
    if pool.index != batch.index:
        raise ValueError("cache and batch must be on one device")


def append(pool: PagedCache, layer: int, batch: Batch, k: torch.Tensor, v: torch.Tensor) -> None:
    """Quantises the new tokens' keys and values ([tokens, kv_heads, D]) into `layer` of the cache."""
    _same_device(pool, batch)
    strides = _packed(k, None, pool.kv_heads, pool, None, "k")
    rows = k.shape[0]
    _int32("layer", layer)
    if _packed(v, rows, pool.kv_heads, pool, k.dtype, "v") != strides:
        raise ValueError("k and v must share their strides")
    _call(pool, _L.ssba_cache_append, "ssba_cache_append", pool.desc, layer, batch.desc(rows), _DTYPES[k.dtype],
          k.data_ptr(), v.data_ptr(), *strides)


def _scratch(size: int, given, pool):
    """(tensor to keep alive, address, bytes) of a workspace."""
    if given is not None:
        if not (isinstance(given, torch.Tensor) and given.get_device() == pool.index and given.is_contiguous()):
            raise ValueError("scratch must be a contiguous GPU tensor on the cache's device")
        return given, given.data_ptr(), given.numel() * given.element_size()
    if size == 0:
        return None, None, 0
    t = torch.empty(size, dtype=torch.uint8, device=pool.device)
    return t, t.data_ptr(), size


def select(pool: PagedCache, layer: int, batch: Batch, q: torch.Tensor, *, keep: int, first: int = 1, last: int = 1,
           causal: bool = True, lists: Optional[torch.Tensor] = None,
           scratch: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The `keep` pages each new token reads: int32 [tokens, kv_heads, 1 + keep] (count, pages of the sequence
    ascending, -1 padding).  `first` leading and `last` trailing pages are always among them."""
    _same_device(pool, batch)
    qs = _packed(q, None, None, pool, None, "q")
    rows, heads, _ = q.shape
    _int32("layer, keep, first or last", layer, keep, first, last)
    b = batch.desc(rows)
    desc = _lib.CacheQuery(heads, _DTYPES[q.dtype], 1 if causal else 0, keep, first, last, 0.0, *qs, 0, 0)
    size = ctypes.c_size_t(0)
    _lib.check(_L.ssba_cache_select_workspace_size(pool.desc, b, desc, size), "ssba_cache_select_workspace_size")
    if lists is None:
        lists = torch.empty((rows, pool.kv_heads, 1 + keep), dtype=torch.int32, device=pool.device)
    else:
        _check(lists, (rows, pool.kv_heads, 1 + keep), torch.int32, pool.index, "lists")
    alive, at, have = _scratch(size.value, scratch, pool)
    _call(pool, _L.ssba_cache_select, "ssba_cache_select", pool.desc, layer, b, desc, q.data_ptr(), lists.data_ptr(),
          lists.numel() * 4, at, have)
    return lists


def _softmax_scale(scale: Optional[float]) -> float:
    """As the library takes it: fp32, where 0 stands for 1 / sqrt(D)."""
    if scale is None:
        return 0.0
    x = ctypes.c_float(scale).value
    if x <= 0.0:
        raise ValueError("scale must be positive in fp32 (None: 1 / sqrt(D))")
    return x


def attend(pool: PagedCache, layer: int, batch: Batch, q: torch.Tensor, *, lists: Optional[torch.Tensor] = None,
           causal: bool = True, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
           scratch: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the new tokens' queries [tokens, heads, D] over what their sequences hold, or over the pages
    that `lists` (of select) names.  scale: positive; None: 1 / sqrt(D).  Rows of no sequence are left as they are
    in `out`."""
    _same_device(pool, batch)
    qs = _packed(q, None, None, pool, None, "q")
    rows, heads, d = q.shape
    _int32("layer", layer)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        os = (heads * d, d)
    else:
        os = _packed(out, rows, heads, pool, q.dtype, "out")
    keep, lp, lb = 0, None, 0
    if lists is not None:
        if not (isinstance(lists, torch.Tensor) and lists.dim() == 3 and lists.shape[2] > 1):
            raise ValueError("lists: expected [tokens, kv_heads, 1 + keep]")
        keep = lists.shape[2] - 1
        _check(lists, (rows, pool.kv_heads, 1 + keep), torch.int32, pool.index, "lists")
        lp, lb = lists.data_ptr(), lists.numel() * 4
    b = batch.desc(rows)
    desc = _lib.CacheQuery(heads, _DTYPES[q.dtype], 1 if causal else 0, keep, 0, 0,
                           _softmax_scale(scale), *qs, *os)
    size = ctypes.c_size_t(0)
    _lib.check(_L.ssba_cache_attend_workspace_size(pool.desc, b, desc, 0 if lists is None else 1, size),
               "ssba_cache_attend_workspace_size")
    alive, at, have = _scratch(size.value, scratch, pool)
    _call(pool, _L.ssba_cache_attend, "ssba_cache_attend", pool.desc, layer, b, desc, q.data_ptr(), lp, lb,
          out.data_ptr(), at, have)
    return out


def _query(pool: PagedCache, layer: int, batch: Batch, q, causal: bool, scale, out):
    """What attention without lists takes: (output, batch, query)."""
    _same_device(pool, batch)
    qs = _packed(q, None, None, pool, None, "q")
    rows, heads, d = q.shape
    _int32("layer", layer)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        os = (heads * d, d)
    else:
        os = _packed(out, rows, heads, pool, q.dtype, "out")
    return out, batch.desc(rows), _lib.CacheQuery(heads, _DTYPES[q.dtype], 1 if causal else 0, 0, 0, 0,
                                                  _softmax_scale(scale), *qs, *os)


def attend_window(pool: PagedCache, layer: int, batch: Batch, q: torch.Tensor, *, window: int, sinks: int = 0,
                  causal: bool = True, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                  scratch: Optional[torch.Tensor] = None) -> torch.Tensor:
    """As `attend` without lists, of the last `window` tokens and the first `sinks`: a token at position p sees j <
    sinks and j > p - window, of what `causal` lets it see.  Pages between the two are not read.  (window.forward:
    the form for rows that are not cached, with gradients.)"""
    out, b, desc = _query(pool, layer, batch, q, causal, scale, out)
    window, sinks = int(window), int(sinks)
    _int32("window or sinks", window, sinks)
    if window < 1 or sinks < 0:
        raise ValueError("window must be 1 or more, sinks 0 or more")
    size = ctypes.c_size_t(0)
    _lib.check(_L.ssba_cache_attend_window_workspace_size(pool.desc, b, desc, window, sinks, size),
               "ssba_cache_attend_window_workspace_size")
    alive, at, have = _scratch(size.value, scratch, pool)
    _call(pool, _L.ssba_cache_attend_window, "ssba_cache_attend_window", pool.desc, layer, b, desc, window, sinks,
          q.data_ptr(), out.data_ptr(), at, have)
    return out


def attend_shared(pool: PagedCache, layer: int, batch: Batch, prefix: Prefix, q: torch.Tensor, *, causal: bool = True,
                  scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                  scratch: Optional[torch.Tensor] = None) -> torch.Tensor:
    """As `attend` without lists, of sequences that share their first pages by groups: these are read once for a
    group, whatever the number of its sequences.  It pays where reading is what takes the time: a few new tokens each;
    for chunks of 64 and more `attend` is as fast or faster."""
    out, b, desc = _query(pool, layer, batch, q, causal, scale, out)
    if not isinstance(prefix, Prefix) or prefix.index != pool.index:
        raise ValueError("prefix: expected a cache.Prefix on the cache's device")
    x = prefix.desc(batch.table.shape[0])
    size = ctypes.c_size_t(0)
    _lib.check(_L.ssba_cache_attend_shared_workspace_size(pool.desc, b, desc, x, size),
               "ssba_cache_attend_shared_workspace_size")
    alive, at, have = _scratch(size.value, scratch, pool)
    _call(pool, _L.ssba_cache_attend_shared, "ssba_cache_attend_shared", pool.desc, layer, b, desc, x, q.data_ptr(),
          out.data_ptr(), at, have)
    return out


def _rows(pool: PagedCache, table, lens, refs) -> _lib.CachePages:
    _gpu_of(table, 2, "table")
    _check(table, None, torch.int32, pool.index, "table")
    _int32("table", *table.shape)
    _check(lens, (table.shape[0],), torch.int32, pool.index, "lens")
    _check(refs, (pool.pages,), torch.int32, pool.index, "refs")
    return _lib.CachePages(table.shape[0], table.shape[1], table.data_ptr(), lens.data_ptr(), refs.data_ptr())


def _pages_scratch(pool: PagedCache, desc, n: int, given):
    size = ctypes.c_size_t(0)
    _lib.check(_L.ssba_pages_workspace_size(pool.desc, desc, n, size), "ssba_pages_workspace_size")
    return _scratch(size.value, given, pool)


def _info(pool: PagedCache, given) -> torch.Tensor:
    if given is None:
        return torch.empty(2, dtype=torch.int32, device=pool.device)
    _check(given, (2,), torch.int32, pool.index, "info")
    return given


def _numbers(pool: PagedCache, t, n, what: str) -> int:
    """Checks a vector of row or page numbers (of length n, if given); its length."""
    _check(t, None, torch.int32, pool.index, what)
    if t.dim() != 1 or (n is not None and t.shape[0] != n):
        raise ValueError(f"{what}: expected a vector" + (f" of {n}" if n is not None else ""))
    _int32(what, t.shape[0])
    return t.shape[0]


def reserve(pool: PagedCache, table, lens, refs, info=None, scratch=None) -> torch.Tensor:
    """Gives every row the pages that lens tokens need, lowest free page first.  Updates table and refs; returns
    info = {entries served, entries left without a page}."""
    desc = _rows(pool, table, lens, refs)
    info = _info(pool, info)
    alive, at, have = _pages_scratch(pool, desc, 0, scratch)
    _call(pool, _L.ssba_pages_reserve, "ssba_pages_reserve", pool.desc, desc, info.data_ptr(), at, have)
    return info


def fork(pool: PagedCache, table, lens, refs, src, dst, info=None, scratch=None) -> torch.Tensor:
    """Row dst[j] becomes a copy of row src[j]: complete pages shared, an incomplete last one copied.  Updates
    table, lens and refs; returns info = {pairs forked, of them cut for lack of a page}."""
    desc = _rows(pool, table, lens, refs)
    n = _numbers(pool, src, None, "src")
    _numbers(pool, dst, n, "dst")
    info = _info(pool, info)
    alive, at, have = _pages_scratch(pool, desc, n, scratch)
    _call(pool, _L.ssba_pages_fork, "ssba_pages_fork", pool.desc, desc, n, src.data_ptr(), dst.data_ptr(),
          info.data_ptr(), at, have)
    return info


def release(pool: PagedCache, table, lens, refs, rows, info=None, scratch=None) -> torch.Tensor:
    """Empties rows.  Updates table, lens and refs; returns info = {entries released, pages that became free}."""
    desc = _rows(pool, table, lens, refs)
    n = _numbers(pool, rows, None, "rows")
    info = _info(pool, info)
    alive, at, have = _pages_scratch(pool, desc, n, scratch)
    _call(pool, _L.ssba_pages_release, "ssba_pages_release", pool.desc, desc, n, rows.data_ptr(), info.data_ptr(), at,
          have)
    return info


def compact(pool: PagedCache, table, refs, table_out=None, refs_out=None, info=None, scratch=None):
    """Moves the pages in use to the low end of the pool.  Returns (table, refs, info) after it, info = {pages in
    use, pages moved}; table_out and refs_out may be table and refs themselves."""
    # lens takes no part: its place is filled by another array
    _gpu_of(table, 2, "table")
    _check(table, None, torch.int32, pool.index, "table")
    _int32("table", *table.shape)
    _check(refs, (pool.pages,), torch.int32, pool.index, "refs")
    desc = _lib.CachePages(table.shape[0], table.shape[1], table.data_ptr(), refs.data_ptr(), refs.data_ptr())
    table_out = torch.empty_like(table) if table_out is None else table_out
    refs_out = torch.empty_like(refs) if refs_out is None else refs_out
    _check(table_out, table.shape, torch.int32, pool.index, "table_out")
    _check(refs_out, refs.shape, torch.int32, pool.index, "refs_out")
    info = _info(pool, info)
    alive, at, have = _pages_scratch(pool, desc, 0, scratch)
    _call(pool, _L.ssba_pages_compact, "ssba_pages_compact", pool.desc, desc, table_out.data_ptr(),
          refs_out.data_ptr(), info.data_ptr(), at, have)
    return table_out, refs_out, info


def copy_pages(pool: PagedCache, src, dst, to: Optional[PagedCache] = None) -> None:
    """Copies pages of all layers, to.pages[dst[j]] = pool.pages[src[j]] (`to`: another cache of the same layout)."""
    to = pool if to is None else to
    if to.index != pool.index:
        raise ValueError("both caches must be on one device")
    n = _numbers(pool, src, None, "src")
    _numbers(pool, dst, n, "dst")
    _call(pool, _L.ssba_pages_copy, "ssba_pages_copy", pool.desc, to.desc, n, src.data_ptr(), dst.data_ptr())
