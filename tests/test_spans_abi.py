"""Refusals of the windowed attention, the rotary positions, the cache's windows and shared prefixes, and of their
bindings (no GPU: every check comes before a launch; tensors that say they are on one)."""
import ctypes
import importlib
import os

import pytest
import torch

from paper_2605_15684_amd import _lib

OK, ARG, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4
P = 0x10000            # an address that is aligned; nothing reads it


@pytest.fixture(scope="module", autouse=True)
def built():
    global L, rope, window, cache
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2605_15684_amd import build
        build.build()
    L = _lib.load()
    rope, window, cache = (importlib.import_module("paper_2605_15684_amd." + x) for x in ("rope", "window", "cache"))


def wdesc(**kw):
    d = dict(batch=1, seq=100, heads=4, kv_heads=2, head_dim=64, dtype=0, window=32, sinks=4, seqs=0, max_len=0,
             softmax_scale=0.0, cu=0)
    d.update(kw)
    w = _lib.WindowDesc()
    for k, v in d.items():
        setattr(w, k, _lib.Strides(*v) if k in "qkvo" else v)
    return w


def forward(w, q=P, k=P, v=P, o=P, lse=P):
    return L.ssba_window_forward(ctypes.byref(w), q, k, v, o, lse, None)


def test_window_refusals():
    bad = [(dict(heads=5), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(seq=-1), SHAPE),
           (dict(head_dim=96), UNSUPPORTED), (dict(dtype=2), ARG), (dict(window=0), ARG), (dict(sinks=-1), ARG),
           (dict(max_len=-1), ARG), (dict(softmax_scale=float("inf")), ARG), (dict(softmax_scale=float("nan")), ARG),
           (dict(seq=(1 << 30) + 1), UNSUPPORTED), (dict(heads=131072, kv_heads=2), UNSUPPORTED),
           (dict(seqs=65536, cu=P), UNSUPPORTED), (dict(seqs=-1), UNSUPPORTED), (dict(seqs=2, batch=2, cu=P), SHAPE),
           (dict(cu=P), SHAPE), (dict(seqs=2), ARG), (dict(seqs=2, cu=P + 2), ARG), (dict(q=(0, 0, 8)), SHAPE),
           (dict(q=(0, 64, 65)), UNSUPPORTED), (dict(k=(0, -64, 64)), SHAPE), (dict(v=(0, 32, 128)), SHAPE),
           (dict(o=(6400, 64, (1 << 20) + 8)), UNSUPPORTED), (dict(batch=1 << 20, heads=64, kv_heads=64), UNSUPPORTED),
           (dict(batch=2, o=(0, 64, 256)), SHAPE)]
    for kw, want in bad:
        assert forward(wdesc(**kw)) == want, kw
    assert L.ssba_window_forward(None, P, P, P, P, P, None) == ARG
    for at in range(4):
        args = [P] * 4
        args[at] = None
        assert forward(wdesc(), *args) == ARG
        args[at] = P + 8
        assert forward(wdesc(), *args) == ARG
    assert forward(wdesc(), lse=P + 2) == ARG
    # nothing to do
    assert forward(wdesc(seq=0), None, None, None, None, None) == OK
    assert forward(wdesc(batch=0), None, None, None, None, None) == OK


def test_window_workspace():
    size = ctypes.c_size_t(0)

    def need(**kw):
        assert L.ssba_window_backward_workspace_size(ctypes.byref(wdesc(**kw)), ctypes.byref(size)) == OK
        return size.value

    rows = lambda n: -(-4 * n // 256) * 256
    assert need(sinks=0) >= 2 * rows(400)
    assert need(seq=0) == 0
    # full chips keep no parts without sinks: two values a row
    assert need(batch=8, seq=16384, sinks=0, heads=16, kv_heads=8) == 2 * rows(8 * 16 * 16384)
    # one tile of sinks, its queries in chunks of 1280 (window 1024 + 128, to a multiple of 128, at least 1024)
    chunk = 1152
    assert need(batch=8, seq=16384, sinks=4, heads=16, kv_heads=8, window=1024) == \
        2 * rows(8 * 16 * 16384) + 64 * -(-16384 // chunk) * 2 * 128 * 64 * 4
    assert L.ssba_window_backward_workspace_size(ctypes.byref(wdesc(window=0)), ctypes.byref(size)) == ARG
    w, g = wdesc(), _lib.WindowGrads()
    full = need()
    call = lambda scratch, n, **kw: L.ssba_window_backward(ctypes.byref(w), ctypes.byref(g), P, P, P, P, P, P, P, P, P,
                                                           scratch, n, None)
    assert call(P, full - 1) == WORKSPACE and call(None, full) == ARG and call(P + 4, full) == ARG
    g.dk = _lib.Strides(0, 32, 64)
    assert call(P, full) == SHAPE
    assert L.ssba_window_backward(ctypes.byref(w), None, P, P, P, P, P, P, P, P, P, P, full, None) == ARG


def turn(n=1, rows=4, batch=1, dtype=0, inverse=0, pos=P, st=3, tensors=None, **kw):
    axis, freq = (ctypes.c_int32 * 64)(*([0] * 64)), (ctypes.c_double * 64)(*([0.5] * 64))
    d = dict(head_dim=64, pairs=0, axes=3)
    d.update(kw)
    if "first_axis" in d:
        axis[0] = d.pop("first_axis")
    if "first_freq" in d:
        freq[0] = d.pop("first_freq")
    r = _lib.RopeDesc(d["head_dim"], d["pairs"], d["axes"], ctypes.addressof(axis), ctypes.addressof(freq))
    arr = (_lib.RopeTensor * 2)()
    for i, t in enumerate(tensors or [dict(), dict()]):
        for k, v in {**dict(heads=2, x=P, y=P), **t}.items():
            setattr(arr[i], k, v)
    return L.ssba_rope_rotate(ctypes.byref(r), dtype, inverse, batch, rows, pos, 0, st, n, ctypes.addressof(arr), None)


def test_rope_refusals():
    for kw, want in [(dict(head_dim=96), UNSUPPORTED), (dict(pairs=2), ARG), (dict(axes=0), UNSUPPORTED),
                     (dict(axes=5), UNSUPPORTED), (dict(first_axis=3), ARG), (dict(first_axis=-2), ARG),
                     (dict(first_freq=float("nan")), ARG), (dict(first_freq=2.0 ** 21), UNSUPPORTED), (dict(dtype=2), ARG),
                     (dict(inverse=2), ARG), (dict(n=0), ARG), (dict(n=3), ARG), (dict(rows=-1), SHAPE),
                     (dict(batch=-1), SHAPE), (dict(st=-1), SHAPE), (dict(pos=None), ARG), (dict(pos=P + 2), ARG),
                     (dict(tensors=[dict(heads=0)]), SHAPE), (dict(tensors=[dict(heads=65537)]), UNSUPPORTED),
                     (dict(tensors=[dict(x=None)]), ARG), (dict(tensors=[dict(x=P + 8)]), ARG),
                     (dict(tensors=[dict(x_stride_t=32)]), SHAPE),
                     (dict(tensors=[dict(x_stride_h=64, x_stride_t=129)]), UNSUPPORTED),
                     (dict(tensors=[dict(x_stride_h=64, x_stride_t=128)]), ARG),      # in place with other strides
                     (dict(tensors=[dict(), dict(heads=0)], n=2), SHAPE),
                     (dict(rows=2 ** 31 - 1, batch=64), UNSUPPORTED)]:
        assert turn(**kw) == want, kw
    assert turn(rows=0, pos=None) == OK and turn(batch=0) == OK


def test_rope_plans():
    p = rope.plan(64, (4, 6), theta=100.0, step=(1.0, 2.0))
    assert list(p._axis) == [0] * 4 + [1] * 6 + [-1] * 22
    assert list(p._freq)[:10] == [100.0 ** -(i / 4) for i in range(4)] + [2.0 * 100.0 ** -(i / 6) for i in range(6)]
    s = rope.plan(64, (4, 6), theta=100.0, spectrum="shared", pairs="halves")
    assert list(s._freq)[:10] == [100.0 ** -(j / 32) for j in range(10)]
    for kw in (dict(sections=(20, 13)), dict(sections=(-1, 3)), dict(sections=(1,), spectrum="x"),
               dict(sections=(1,), theta=0.0), dict(sections=(1,), theta=float("nan")), dict(sections=(1, 1), step=(1.0,)),
               dict(sections=(1,), pairs="x"), dict(sections=()), dict(sections=(1,) * 5), dict(head_dim=96, sections=(1,)),
               dict(sections=(1,), step=(2.0 ** 30,))):
        with pytest.raises(ValueError):
            rope.plan(kw.pop("head_dim", 64), **kw)
    with pytest.raises(ValueError):
        rope.Plan(64, 1, [0] * 31, [1.0] * 31)
    with pytest.raises(ValueError):
        rope.Plan(64, 1, [1] * 32, [1.0] * 32)


class OnGpu(torch.Tensor):
    """A host tensor that says it is on GPU 0."""
    is_cuda = True

    def get_device(self):
        return 0


def gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def test_rope_binding():
    plan, q, pos = rope.plan(64, (8, 8)), gpu(5, 4, 64), gpu(5, 2, dtype=torch.int32)
    for args, kw in [((None, pos, q), {}), ((plan, pos, torch.zeros(5, 4, 64, dtype=torch.bfloat16)), {}),
                     ((plan, pos, gpu(5, 4, 64, dtype=torch.float16)), {}), ((plan, pos, gpu(5, 4, 128)), {}),
                     ((plan, pos, gpu(5, 64)), {}), ((plan, pos.long(), q), {}), ((plan, pos[:4], q), {}),
                     ((plan, gpu(5, 3, dtype=torch.int32), q), {}), ((plan, gpu(2, 5, dtype=torch.int32).T, q), {}),
                     ((plan, pos, q, gpu(4, 2, 64)), {}), ((plan, pos, q, gpu(5, 2, 64, dtype=torch.float32)), {}),
                     ((plan, pos, q), dict(k_out=q)), ((plan, pos, q), dict(q_out=gpu(5, 3, 64))),
                     ((plan, pos, q[:1].expand(5, 4, 64)), {}), ((plan, pos, gpu(5, 4, 128)[..., ::2]), {}),
                     ((plan, pos, gpu(1, 4, 5, 64)[:, :, :4]), {}),
                     ((plan, gpu(3, 5, 2, dtype=torch.int32), gpu(2, 4, 5, 64)), {})]:
        with pytest.raises(ValueError):
            rope.rotate(*args, **kw)


def test_window_binding():
    q, k = gpu(2, 4, 9, 64), gpu(2, 2, 9, 64)
    pq, pk, cu = gpu(9, 4, 64), gpu(9, 2, 64), gpu(3, dtype=torch.int32)
    ok = dict(window=4)
    for args, kw in [((torch.zeros(2, 4, 9, 64), k, k), ok), ((q, k, k[:, :1]), ok), ((q, gpu(2, 3, 9, 64), k), ok),
                     ((q, k.float(), k), ok), ((q, k, k), dict(window=0)), ((q, k, k), dict(window=4, sinks=-1)),
                     ((q, k, k), dict(window=4, scale=0.0)), ((q, k, k), dict(window=4, scale=float("nan"))),
                     ((q, k, k), dict(window=1 << 31)), ((q, k, k), dict(window=4, sinks=1 << 31)),
                     ((q, k, k), dict(window=4, cu=cu)), ((pq, pk, pk), ok), ((pq, pk, pk), dict(window=4, cu=cu.long())),
                     ((pq, pk, pk), dict(window=4, cu=cu[:1])), ((q, k, k), dict(window=4, out=gpu(2, 4, 8, 64))),
                     ((q[:, :1].expand(2, 4, 9, 64), k, k), ok), ((gpu(2, 4, 9, 128)[..., ::2], k, k), ok),
                     ((q, k, k), dict(window=4, lse=gpu(2, 4, 8, dtype=torch.float32)))]:
        with pytest.raises(ValueError):
            window.forward(*args, **kw)
    lse = gpu(2, 4, 9, dtype=torch.float32)
    for bad in (dict(dout=q.float()), dict(dq=gpu(2, 4, 8, 64)), dict(dk=q), dict(lse=lse[:1]),
                dict(scratch=torch.zeros(1 << 20, dtype=torch.uint8))):
        kw = {**dict(dout=q, lse=lse), **bad}
        with pytest.raises(ValueError):
            window.backward(q, k, k, q, kw.pop("dout"), kw.pop("lse"), window=4, **kw)


def test_cache_span_refusals():
    c = _lib.CacheDesc(1, 8, 2, 64, 16, P, P, P, P)
    b = _lib.CacheBatch(2, 4, 2, 1, 0, P, P, P)
    q = _lib.CacheQuery(4, 0, 1, 0, 0, 0, 0.0, 0, 0, 0, 0)
    size = ctypes.c_size_t(0)
    attend = lambda win, sinks, scratch=P, n=1 << 40: L.ssba_cache_attend_window(c, 0, b, q, win, sinks, P, P, scratch, n, None)
    for win, sinks in ((0, 0), (-1, 0), (5, -1)):
        assert attend(win, sinks) == ARG
        assert L.ssba_cache_attend_window_workspace_size(c, b, q, win, sinks, size) == ARG
    assert L.ssba_cache_attend_window(c, 1, b, q, 5, 0, P, P, P, 1 << 40, None) == ARG
    assert L.ssba_cache_attend_window(c, 0, b, q, 5, 0, None, P, P, 1 << 40, None) == ARG
    long = _lib.CacheBatch(1, 1 << 16, 1, 1, 0, P, P, P)
    assert L.ssba_cache_attend_window_workspace_size(c, long, q, 1 << 19, 0, size) == OK and size.value > 0
    assert L.ssba_cache_attend_window(c, 0, long, q, 1 << 19, 0, P, P, P, size.value - 1, None) == WORKSPACE
    assert L.ssba_cache_attend_window(c, 0, long, q, 1 << 19, 0, P, P, None, size.value, None) == ARG
    x = lambda *a: _lib.CachePrefix(*a)
    shared = lambda pre, n=1 << 40: L.ssba_cache_attend_shared(c, 0, b, q, pre, P, P, P, n, None)
    for pre, want in ((x(0, 1, 0, P, P), SHAPE), (x(1, 0, 0, P, P), SHAPE), (x(1, 1, -1, P, P), SHAPE),
                      (x(65536, 1, 0, P, P), UNSUPPORTED), (x(1, 65536, 0, P, P), UNSUPPORTED), (x(1, 1, 0, None, P), ARG),
                      (x(1, 1, 0, P, P + 2), ARG), (x(1, 1, 0, P, P), WORKSPACE)):
        assert shared(pre, 0 if want == WORKSPACE else 1 << 40) == want
    assert L.ssba_cache_attend_shared(c, 0, b, q, None, P, P, P, 0, None) == ARG
    i32 = lambda *n: gpu(*n, dtype=torch.int32)
    for first, pages, kw in [(i32(1), i32(1), {}), (i32(3), i32(1), {}), (i32(3).long(), i32(2), {}), (i32(3), i32(2), dict(max_seqs=0)),
                             (i32(3), i32(2), dict(max_len=-1)), (i32(3), i32(2), dict(max_seqs=1 << 31)),
                             (torch.zeros(3, dtype=torch.int32), i32(2), {})]:
        with pytest.raises(ValueError):
            cache.Prefix(first, pages, **kw)
