"""Rotary positions, windowed attention and the cache as they are used: a generation step captured and replayed, the
two forms of the window against each other, other streams, calls at once, gradients by differences, large tensors."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C

from _cache import gpu_batch, host_pool, rounded
from _window import BF16, F32, U, normal

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_a_generation_step_captured_and_replayed():
    """rotate, append, attend_window and attend_shared of four sequences in one graph; positions, lengths and rows
    change between replays, with eager work of the same program between them."""
    from paper_2605_15684_amd import cache, rope
    rng = np.random.default_rng(1)
    page, d, heads, kv, seqs, most = 16, 64, 8, 2, 4, 6
    plan = rope.plan(d, (8, 12, 12))
    data = lambda *s: normal(rng, s, BF16).cuda()

    def make():
        torch.manual_seed(0)
        pool = cache.alloc(1, 80, kv, d, page)
        table = torch.arange(80, dtype=torch.int32, device="cuda").view(seqs, 20).clone()
        table[:, :2] = table[0, :2]                       # two shared pages
        return pool, table, torch.zeros(seqs, dtype=torch.int32, device="cuda")

    prompt = data(32, kv, d), data(32, kv, d)
    steps = [([2, 1, 0, 3], [5, 9, 0, 2]), ([1, 1, 1, 1], [0, 1, 2, 3]), ([0, 6, 0, 0], [0, 7, 0, 0]), ([1, 0, 2, 3], [4, 0, 4, 4]),
             ([3, 3, 0, 0], [9, 8, 0, 0])]
    rows = most * seqs
    inputs = [(data(rows, heads, d), data(rows, kv, d), data(rows, kv, d), rng.integers(0, 10 ** 5, (rows, 3))) for _ in steps]

    def fill(pool, table):
        batch = cache.Batch(table[:1].contiguous(), ints([32]), ints([0, 32]), 32)
        cache.append(pool, 0, batch, *prompt)

    def step(pool, table, lens, cu, pos, q, k, v, prefix, outs):
        rope.rotate(plan, pos, q, k, q_out=q, k_out=k)
        batch = cache.Batch(table, lens, cu, most)
        cache.append(pool, 0, batch, k, v)
        cache.attend_window(pool, 0, batch, q, window=20, sinks=3, out=outs[0])
        cache.attend_shared(pool, 0, batch, prefix, q, out=outs[1])

    def run(captured):
        pool, table, lens = make()
        fill(pool, table)
        prefix = cache.Prefix(ints([0, seqs]), ints([2]), seqs, 32)
        lens += 32
        cu, pos = ints([0] * (seqs + 1)), ints([[0, 0, 0]] * rows)
        q, k, v = (torch.zeros_like(x) for x in inputs[0][:3])
        outs = [torch.full_like(q, 3.0) for _ in range(2)]
        held = lens.clone()
        if captured:
            lens.copy_(held)
            step(pool, table, lens, cu, pos, q, k, v, prefix, outs)      # no new tokens: nothing but a warm-up
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step(pool, table, lens, cu, pos, q, k, v, prefix, outs)
        results = []
        for (news, _), (qi, ki, vi, pi) in zip(steps, inputs):
            held = held + ints(news)
            lens.copy_(held)
            cu.copy_(ints(np.concatenate([[0], np.cumsum(news)]).tolist()))
            pos.copy_(torch.from_numpy(pi.astype(np.int32)))
            for dst, src in ((q, qi), (k, ki), (v, vi)):
                dst.copy_(src)
            for o in outs:
                o.fill_(3.0)
            if captured:
                graph.replay()
            else:
                step(pool, table, lens, cu, pos, q, k, v, prefix, outs)
            torch.cuda.synchronize()
            results.append([o.clone() for o in outs] + [q.clone(), pool.k.view(torch.uint8).clone()])
        return results, host_pool(pool), table.cpu().numpy()

    eager, pool, table = run(False)
    replayed, _, _ = run(True)
    for a, b in zip(eager, replayed):
        for x, y in zip(a[:3], b[:3]):
            assert torch.equal(x, y)
    for (news, _), outs in zip(steps, eager):
        for o in outs[:2]:
            assert (o[sum(news):] == 3.0).all(), "rows of no sequence were written"
    # the last step against the oracle
    news = steps[-1][0]
    held = 32 + np.sum([n for n, _ in steps], axis=0)
    batch = (table, held.astype(np.int32), np.concatenate([[0], np.cumsum(news)]).astype(np.int32))
    q64 = eager[-1][2][:sum(news)].double().cpu().numpy()
    from test_gpu_cache import check_attend
    check_attend(eager[-1][0][:sum(news)], C.attend_window(pool, 0, batch, q64, page, 20, 3), 64, d, BF16)
    check_attend(eager[-1][1][:sum(news)], C.attend(pool, 0, batch, q64, page), 64, d, BF16)


def test_the_two_forms_of_the_window_agree():
    """Tokens appended to a cache and attended there, against window.forward of the values that the cache holds."""
    from paper_2605_15684_amd import cache, window
    rng = np.random.default_rng(2)
    page, d, heads, kv, n, win, sinks = 32, 128, 6, 2, 300, 70, 5
    pool = cache.alloc(1, 12, kv, d, page)
    table = ints([list(range(11))])
    k, v, q = (normal(rng, (n, h, d), F32).cuda() for h in (kv, kv, heads))
    outs, at = [], 0
    for new in (100, 1, 1, 30, 64, 1, 103):
        batch = cache.Batch(table, ints([at + new]), ints([0, new]), new)
        cache.append(pool, 0, batch, k[at:at + new], v[at:at + new])
        outs.append((at, new, cache.attend_window(pool, 0, batch, q[at:at + new], window=win, sinks=sinks)))
        at += new
    # what the cache holds at the end is what the last call saw
    p = host_pool(pool)
    held = [np.stack([np.concatenate([C.rows_of(p, 0, i, h, w, page, d) for i in range(11)])[:n] for h in range(kv)], 1)
            for w in (0, 1)]
    dk, dv = (torch.from_numpy(x.astype(np.float32)).cuda() for x in held)
    want, _ = window.forward(q, dk, dv, window=win, sinks=sinks, cu=ints([0, n]))
    begin, new, got = outs[-1]
    # both are fp32 sums of the same numbers: |scores| < 8 times 2^-18, sums of 75 values below 8
    assert ((got - want[begin:begin + new]).abs() < 2 ** -14).all()


def test_a_training_step_in_a_graph():
    """rotate, forward, backward, gradients turned back: captured and replayed over new inputs, eager steps between."""
    from paper_2605_15684_amd import rope, window
    rng = np.random.default_rng(3)
    h, kv, d = 4, 2, 64
    plan = rope.plan(d, (16, 16), pairs="halves")
    for dtype in (BF16, F32):
        lens_of = [[700, 1300], [2000, 0], [3, 1997], [0, 1111]]
        rows = 2000
        batches = [[normal(rng, (rows, x, d), dtype).cuda() for x in (h, kv, kv, h)] +
                   [ints(rng.integers(0, 3000, (rows, 2)).tolist()), ints([0, a, a + b])] for a, b in lens_of]
        static = [t.clone() for t in batches[0]]
        kw = dict(window=90, sinks=4, max_len=2000)

        def step(q, k, v, do, pos, cu, outs):
            rq, rk = rope.rotate(plan, pos, q, k)
            o, lse = window.forward(rq, rk, v, cu=cu, out=outs[0], **kw)
            dq, dk, dv = window.backward(rq, rk, v, o, do, lse, cu=cu, dq=outs[1], dk=outs[2], dv=outs[3], **kw)
            rope.rotate(plan, pos, dq, dk, inverse=True, q_out=dq, k_out=dk)

        make = lambda: [torch.zeros_like(static[0]), torch.zeros_like(static[0]), torch.zeros_like(static[1]),
                        torch.zeros_like(static[1])]
        outs = make()
        step(*static, outs)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(*static, outs)
        for b in batches + batches[:1]:
            want = make()
            step(*b, want)                                # eager, the library's own scratch between replays
            for dst, src in zip(static, b):
                dst.copy_(src)
            for o in outs:
                o.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip(outs, want):
                assert torch.equal(x, y)


def test_two_streams_at_once():
    """The same calls on two streams of their own, with scratch of their own, give what one after the other gives."""
    from paper_2605_15684_amd import cache, window
    rng = np.random.default_rng(4)
    d, h, kv, n = 128, 8, 2, 1500
    sets = [[normal(rng, (1, x, n, d), BF16).cuda() for x in (h, kv, kv, h)] for _ in range(2)]
    kw = dict(window=100, sinks=70)

    def train(q, k, v, do):
        o, lse = window.forward(q, k, v, **kw)
        return (o,) + window.backward(q, k, v, o, do, lse, **kw)

    want = [train(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        for s, x in zip(streams, sets):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(train(*x))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        for x, y in zip(g, want[i % 2]):
            assert torch.equal(x, y)


def test_gradients_by_differences():
    """sum(do * o) along a direction changes by what dq, dk and dv say.  In fp32 with a step of 2^-6 the third order is
    below 2^-12 of the second's scale; both sides' fp32 sums of 4 * 90 * 64 terms below 2^-15 of theirs."""
    from paper_2605_15684_amd import window
    rng = np.random.default_rng(5)
    h, kv, d, n = 2, 1, 64, 90
    q, do = (normal(rng, (1, h, n, d), F32).cuda() for _ in range(2))
    k, v = (normal(rng, (1, kv, n, d), F32).cuda() for _ in range(2))
    kw = dict(window=17, sinks=2)
    o, lse = window.forward(q, k, v, **kw)
    grads = window.backward(q, k, v, o, do, lse, **kw)
    f = lambda *x: float((window.forward(*x, **kw)[0].double() * do.double()).sum())
    for i in range(3):
        for seed in range(3):
            g = torch.Generator(device="cuda").manual_seed(seed)
            direction = torch.randn((q, k, v)[i].shape, generator=g, device="cuda")
            direction /= direction.norm()
            x = [q, k, v]
            step = 2.0 ** -6
            up, down = list(x), list(x)
            up[i], down[i] = x[i] + step * direction, x[i] - step * direction
            want = float((grads[i].double() * direction.double()).sum())
            scale = float(grads[i].double().norm())
            assert abs((f(*up) - f(*down)) / (2 * step) - want) < 2.0 ** -9 * scale


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_past_32_bits(dtype):
    """Packed rows whose last ones lie beyond 4 GB: the last sequence's results are those of its rows alone."""
    from paper_2605_15684_amd import rope, window
    d, h, kv, n = 128, 16, 16, 700
    size = 2 if dtype == BF16 else 4
    rows = -(-((1 << 32) + (1 << 28)) // (h * d * size))
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    rng = np.random.default_rng(6)
    data = [torch.empty((rows, h, d), dtype=dtype, device="cuda") for _ in range(4)]
    tail = [normal(rng, (n, h, d), dtype).cuda() for _ in range(4)]
    for x, y in zip(data, tail):
        x[rows - n:] = y
    kw = dict(window=100, sinks=3)
    cu = ints([rows - n, rows])
    o, lse = window.forward(*data[:3], cu=cu, **kw)
    grads = window.backward(*data[:3], o, data[3], lse, cu=cu, **kw)
    alone = ints([0, n])
    wo, wl = window.forward(*tail[:3], cu=alone, **kw)
    wg = window.backward(*tail[:3], wo, tail[3], wl, cu=alone, **kw)
    assert torch.equal(o[rows - n:], wo) and torch.equal(lse[:, rows - n:], wl)
    for x, y in zip(grads, wg):
        assert torch.equal(x[rows - n:], y)
    del grads, o
    plan = rope.plan(d, (32, 32))
    pos = torch.zeros((rows, 2), dtype=torch.int32, device="cuda")
    pos[rows - n:, 0] = torch.arange(n, device="cuda")
    pos[rows - n:, 1] = 3
    assert torch.equal(rope.rotate(plan, pos, data[0])[rows - n:], rope.rotate(plan, pos[rows - n:], tail[0]))


def test_no_rows():
    from paper_2605_15684_amd import cache, rope, window
    q = torch.zeros((0, 4, 64), dtype=BF16, device="cuda")
    o, lse = window.forward(q, q, q, window=3, cu=ints([0, 0]))
    assert o.shape == q.shape and lse.shape == (4, 0)
    assert window.backward(q, q, q, o, q, lse, window=3, cu=ints([0, 0]))[0].shape == q.shape
    q4 = torch.zeros((2, 4, 0, 64), dtype=BF16, device="cuda")
    o, lse = window.forward(q4, q4, q4, window=3)
    window.backward(q4, q4, q4, o, q4, lse, window=3)
    plan = rope.plan(64, (4,))
    assert rope.rotate(plan, torch.zeros((0, 1), dtype=torch.int32, device="cuda"), q).shape == q.shape
    pool = cache.alloc(1, 2, 4, 64, 16)
    batch = cache.Batch(ints([[0, 1]]), ints([0]), ints([0, 0]), 1)
    assert cache.attend_window(pool, 0, batch, q, window=3).shape == q.shape
    prefix = cache.Prefix(ints([0, 1]), ints([0]))
    assert cache.attend_shared(pool, 0, batch, prefix, q).shape == q.shape
    # rows, but none of a sequence
    q = torch.zeros((3, 4, 64), dtype=BF16, device="cuda")
    out = torch.full_like(q, 2.0)
    cache.attend_shared(pool, 0, batch, prefix, q, out=out)
    cache.attend_window(pool, 0, batch, q, window=3, out=out)
    o, lse = window.forward(q, q, q, window=3, cu=ints([0, 0, 0]), out=out)
    window.backward(q, q, q, o, q, lse, window=3, cu=ints([0, 0, 0]), dq=out)
    assert (out == 2.0).all()


@pytest.mark.parametrize("cu", [[-5, 3, 100], [0, 40, 20, 60], [60, 0], [2 ** 31 - 1, -2 ** 31, 7], [10, 10, 10]])
def test_whatever_cu_holds(cu):
    """Nothing leaves the arrays: what lies around them keeps its values."""
    from paper_2605_15684_amd import window
    rows, d = 64, 64
    big = torch.full((rows + 256, 2, d), 9.0, dtype=BF16, device="cuda")
    inner = lambda: big.clone()
    q, k, v, do = (torch.zeros((rows, 2, d), dtype=BF16, device="cuda") for _ in range(4))
    held = [inner() for _ in range(4)]
    o, dq, dk, dv = (x[128:128 + rows] for x in held)
    kw = dict(window=7, sinks=70, cu=ints(cu))
    lse_all = torch.full((4, rows), 9.0, device="cuda")
    lse = lse_all[1:3]
    window.forward(q, k, v, out=o, lse=lse, **kw)
    window.backward(q, k, v, o, do, lse, dq=dq, dk=dk, dv=dv, **kw)
    torch.cuda.synchronize()
    for x in held:
        assert (x[:128] == 9.0).all() and (x[128 + rows:] == 9.0).all()
    assert (lse_all[0] == 9.0).all() and (lse_all[3] == 9.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_shared_tiles_in_a_graph_and_twice(dtype):
    """Few rows of a long window (the tiles of a workgroup go to two groups of waves): the same bits in every run, eager,
    captured and on another stream."""
    from paper_2605_15684_amd import window
    rng = np.random.default_rng(11)
    cu = ints([2, 300, 300, 771])
    q, do = (normal(rng, (775, 4, 64), dtype).cuda() for _ in range(2))
    k, v = (normal(rng, (775, 2, 64), dtype).cuda() for _ in range(2))
    kw = dict(window=256, sinks=3, cu=cu)

    def run(out):
        o, lse = window.forward(q, k, v, out=out[0], lse=out[1], **kw)
        window.backward(q, k, v, o, do, lse, dq=out[2], dk=out[3], dv=out[4], **kw)

    room = lambda: [torch.zeros_like(q), torch.zeros((4, 775), device="cuda")] + [torch.zeros_like(x) for x in (q, k, v)]
    want, other, held = room(), room(), room()
    run(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(other)
    run(held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(held)
    for _ in range(3):
        for x in held:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y, z in zip(held, want, other):
            assert torch.equal(x, y) and torch.equal(z, y)
