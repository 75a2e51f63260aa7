"""Rotary positions with several axes on the GPU against the fp64 oracle (oracle/window_oracle.py).

A turned value a cos - b sin: cosine and sine are rounded to fp32 (their series are exact to 2^-32), so is one product,
and so is the sum: off by 4 * 2^-24 (|a| + |b|) in all, of which a far position's angle takes its part (2^-53 |phi|, phi
below 2^27 here), then half a step of the result's type."""
import numpy as np
import pytest
import torch

from oracle import window_oracle as W

from _window import BF16, F32, U, half, normal

pytestmark = pytest.mark.gpu


def check(got, x, pos, plan_args, inverse, dtype):
    axis, freq, halves = plan_args
    want = W.rotate(x, pos, axis, freq, halves, inverse)
    d = x.shape[-1]
    partner = np.concatenate([x[..., d // 2:], x[..., :d // 2]], -1) if halves else \
        x.reshape(x.shape[:-1] + (d // 2, 2))[..., ::-1].reshape(x.shape)
    bound = half(dtype) * np.abs(want) + 4 * U * (np.abs(x) + np.abs(partner)) + 1e-30
    err = np.abs(got - want)
    assert (err <= bound).all(), (np.argwhere(~(err <= bound))[:4], err.max())


def tables(d, sections, theta, spectrum):
    axis, freq = [-1] * (d // 2), [0.0] * (d // 2)
    j = 0
    for a, n in enumerate(sections):
        for i in range(n):
            axis[j], freq[j] = a, theta ** -(i / n if spectrum == "axis" else j / (d // 2))
            j += 1
    return axis, freq


CASES = [  # rows, heads, kv heads, D, sections, spectrum, pairs, dtype, furthest position
    (1, 1, 1, 64, (32,), "axis", "adjacent", BF16, 10),
    (3, 5, 2, 128, (16, 24, 24), "axis", "adjacent", BF16, 1 << 20),
    (4, 16, 4, 128, (16, 24, 24), "shared", "halves", BF16, 1 << 20),
    (5, 3, 3, 64, (0, 16, 16), "axis", "halves", F32, 4096),
    (17, 24, 8, 128, (10, 11), "axis", "adjacent", F32, 1 << 26),
    (1031, 2, 1, 64, (8, 8, 8, 8), "shared", "adjacent", BF16, 100),
    (600, 7, 1, 128, (64,), "axis", "halves", F32, 1 << 26),
    (2, 64, 64, 64, (1, 0, 2), "axis", "halves", BF16, 1000),
]


@pytest.mark.parametrize("rows,h,kv,d,sections,spectrum,pairs,dtype,far", CASES)
@pytest.mark.parametrize("inverse", [False, True])
def test_packed(rows, h, kv, d, sections, spectrum, pairs, dtype, far, inverse):
    from paper_2605_15684_amd import rope
    rng = np.random.default_rng(rows + h)
    plan = rope.plan(d, sections, theta=10000.0, spectrum=spectrum, pairs=pairs)
    args = tables(d, sections, 10000.0, spectrum) + (pairs == "halves",)
    pos = rng.integers(-far, far + 1, (rows, len(sections))).astype(np.int32)
    q, k = normal(rng, (rows, h, d), dtype), normal(rng, (rows, kv, d), dtype)
    a, b = rope.rotate(plan, torch.from_numpy(pos).cuda(), q.cuda(), k.cuda(), inverse=inverse)
    check(a.double().cpu().numpy(), q.double().numpy(), pos, args, inverse, dtype)
    check(b.double().cpu().numpy(), k.double().numpy(), pos, args, inverse, dtype)
    alone = rope.rotate(plan, torch.from_numpy(pos).cuda(), q.cuda(), inverse=inverse)
    assert torch.equal(alone, a)
    # in place
    x, y = q.cuda(), k.cuda()
    rope.rotate(plan, torch.from_numpy(pos).cuda(), x, y, inverse=inverse, q_out=x, k_out=y)
    assert torch.equal(x, a) and torch.equal(y, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_batches_and_strides(dtype):
    """[B, H, T, D] views of one projection; positions shared by the batch or its own."""
    from paper_2605_15684_amd import rope
    rng = np.random.default_rng(4)
    b, n, h, kv, d = 3, 37, 4, 2, 64
    plan = rope.plan(d, (10, 12, 10), step=(0.5, 1.0, 2.0))
    axis, freq = tables(d, (10, 12, 10), 10000.0, "axis")
    freq = [f * (0.5, 1.0, 2.0)[a] for a, f in zip(axis, freq)]
    proj = normal(rng, (b, n, h + 2 * kv, d), dtype)
    dev = proj.cuda()
    q, k, _ = (x.transpose(1, 2) for x in dev.split([h, kv, kv], 2))
    for shape in ((n, 3), (b, n, 3)):
        pos = rng.integers(0, 500, shape).astype(np.int32)
        out = rope.rotate(plan, torch.from_numpy(pos).cuda(), q, k)
        for x, got in zip((q, k), out):
            for s in range(b):
                check(got[s].double().cpu().numpy().transpose(1, 0, 2), x[s].double().cpu().numpy().transpose(1, 0, 2),
                      pos if len(shape) == 2 else pos[s], (axis, freq, False), False, dtype)
    rope.rotate(plan, torch.from_numpy(pos).cuda(), q, k, q_out=q, k_out=k)     # in place, in the projection
    assert torch.equal(q, out[0]) and torch.equal(k, out[1])
    assert torch.equal(dev[:, :, h + kv:].cpu(), proj[:, :, h + kv:])


def test_pairs_that_stay_keep_everything():
    from paper_2605_15684_amd import rope
    plan = rope.plan(64, (3,))
    x = torch.randn(5, 2, 64, device="cuda")
    x[..., 7] = float("inf")
    x[..., 9] = float("nan")
    x[..., 11] = -0.0
    y = rope.rotate(plan, torch.full((5, 1), 7, dtype=torch.int32, device="cuda"), x)
    assert torch.equal(y[..., 6:].view(torch.int32), x[..., 6:].view(torch.int32))


def test_gradient_by_differences():
    """sum(w * rotate(x)) changes by dx times what rotate(w, inverse) says; linear, so large steps are exact enough."""
    from paper_2605_15684_amd import rope
    rng = np.random.default_rng(8)
    plan = rope.plan(64, (16, 16), pairs="halves")
    pos = torch.from_numpy(rng.integers(0, 5000, (9, 2)).astype(np.int32)).cuda()
    x, w = (normal(rng, (9, 2, 64), F32).cuda() for _ in range(2))
    grad = rope.rotate(plan, pos, w, inverse=True).double()
    f = lambda t: float((w.double() * rope.rotate(plan, pos, t).double()).sum())
    for at in [(0, 0, 0), (3, 1, 31), (8, 0, 32), (5, 1, 63)]:
        up, down = x.clone(), x.clone()
        up[at] += 1.0
        down[at] -= 1.0
        # both sums hold 2 * 64 terms of the row that moved by up to 4 U (|a| + |b|) |w| each; |x| < 8, |w| < 8
        assert abs((f(up) - f(down)) / 2 - float(grad[at])) < 2 * 4 * U * 20 * 8 + 1e-9


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
def test_fp32_rows_may_begin_anywhere(d, pairs):
    """Rows at odd multiples of 4 bytes: the values of aligned ones, and nothing beside them is written."""
    from paper_2605_15684_amd import rope
    n, h, kv = 9, 3, 2
    g = torch.Generator(device="cuda").manual_seed(d)
    plan = rope.plan(d, (d // 4, d // 4), pairs=pairs)
    pos = torch.randint(0, 900, (n, 2), generator=g, device="cuda", dtype=torch.int32)
    wide = lambda heads: torch.randn((n, heads, d + 3), generator=g, device="cuda")
    q, k, q_to, k_to = wide(h), wide(kv), wide(h), wide(kv)
    before = [x.clone() for x in (q_to, k_to)]
    mid = lambda x: x[..., 1:1 + d]
    want = rope.rotate(plan, pos, mid(q).contiguous(), mid(k).contiguous())
    rope.rotate(plan, pos, mid(q), mid(k), q_out=mid(q_to), k_out=mid(k_to))
    for got, y, old in zip((q_to, k_to), want, before):
        assert torch.equal(mid(got), y)
        assert torch.equal(got[..., 0], old[..., 0]) and torch.equal(got[..., 1 + d:], old[..., 1 + d:])
    rope.rotate(plan, pos, mid(q), mid(k), q_out=mid(q), k_out=mid(k))
    assert torch.equal(mid(q), want[0]) and torch.equal(mid(k), want[1])
