"""Gradients of packed sequences under every hint about their lengths: max_len decides which tiles of keys are cut into
chunks and how many workgroups share them, never what comes out beyond the rounding of partial sums."""
import ctypes

import numpy as np
import pytest
import torch

from _window import BF16, F32, check, grouped, normal

pytestmark = pytest.mark.gpu

CASES = [  # lengths, heads, kv heads, D, window, sinks, dtype
    ([1, 1200, 77, 1030], 2, 1, 64, 90, 5, BF16),
    ([1, 1200, 77, 1030], 2, 1, 128, 90, 5, BF16),
    ([1300, 40, 0, 1], 2, 2, 64, 300, 130, F32),
    ([64, 1290], 1, 1, 128, 200, 3, F32),
    ([5, 0, 130, 1, 64], 4, 2, 128, 50, 4, BF16),
    ([33, 2, 97, 400], 6, 2, 128, 300, 2, F32),
    ([900, 3], 4, 1, 128, 700, 0, BF16),
    ([700, 128, 129], 3, 1, 64, 500, 1, F32),
]


def scratch_of(q, k, kw, hint):
    from paper_2605_15684_amd import _lib, window as mod
    size = ctypes.c_size_t(0)
    desc = mod._desc(q, k, k, None, kw["window"], kw["sinks"], None, kw["cu"], hint)
    _lib.check(_lib.load().ssba_window_backward_workspace_size(desc, size), "size")
    return size.value


@pytest.mark.parametrize("lens,h,kv,d,window,sinks,dtype", CASES)
def test_gradients_under_every_hint(lens, h, kv, d, window, sinks, dtype):
    from paper_2605_15684_amd import window as mod
    rng = np.random.default_rng(sum(lens) + d + h)
    rows = sum(lens)
    q, do = (normal(rng, (rows, h, d), dtype) for _ in range(2))
    k, v = (normal(rng, (rows, kv, d), dtype) for _ in range(2))
    at = np.concatenate([[0], np.cumsum(lens)])
    cu = torch.from_numpy(at.astype(np.int32)).cuda()
    dev = [t.cuda() for t in (q, k, v, do)]
    kw = dict(window=window, sinks=sinks, cu=cu)
    refs = {s: grouped(*(t[at[s]:at[s] + n].double().numpy().transpose(1, 0, 2) for t in (q, k, v, do)), window, sinks, dtype)
            for s, n in enumerate(lens) if n}
    sizes = set()
    for hint in (None, 1, 64, 300, max(lens), 10 ** 6, 2 ** 31 - 1):
        o, lse = mod.forward(*dev[:3], **kw, max_len=hint)
        grads = mod.backward(*dev[:3], o, dev[3], lse, **kw, max_len=hint)
        sizes.add(scratch_of(dev[0], dev[1], kw, hint))
        for s, ref in refs.items():
            mine = slice(at[s], at[s + 1])
            for name, t in zip(("o", "dq", "dk", "dv"), (o,) + grads):
                check(name, t[mine].transpose(0, 1), *ref[name])
    if max(lens) > 1152 and sinks:      # a hint of less leaves the tiles of sinks whole
        assert len(sizes) > 1
