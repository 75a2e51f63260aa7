"""Pools and batches for the cache tests: made on the host, mirrored on the GPU."""
import numpy as np
import torch

from oracle import cache_oracle as C


def make_pool(rng, layers, pages, kv, d, page, nan_free=True, scales=(-9, -6)):
    """Random codes with power-of-two scales; kmean random bf16 values."""
    codes = lambda: rng.integers(0, 256, (layers, pages, kv, page * d)).astype(np.uint8)
    pool = {"k": codes(), "v": codes()}
    if nan_free:
        for x in ("k", "v"):
            pool[x][(pool[x] & 127) == 127] &= 0xFE
    pool["scale"] = (2.0 ** rng.integers(scales[0], scales[1] + 1, (layers, pages, kv, 2))).astype(np.float32)
    pool["kmean"] = C.to_bf16(rng.standard_normal((layers, pages, kv, d)).astype(np.float32))
    return pool


def gpu_pool(pool):
    from paper_2605_15684_amd import cache
    t = {x: torch.from_numpy(pool[x].copy()).to("cuda") for x in pool}
    return cache.PagedCache(t["k"].view(torch.float8_e4m3fn), t["v"].view(torch.float8_e4m3fn), t["scale"],
                            t["kmean"].to(torch.bfloat16))


def host_pool(p):
    return {"k": p.k.view(torch.uint8).cpu().numpy(), "v": p.v.view(torch.uint8).cpu().numpy(),
            "scale": p.scale.cpu().numpy(), "kmean": p.kmean.float().cpu().numpy()}


def assert_same_pool(got, want):
    for x in ("k", "v"):
        a, b = got[x], want[x]
        nan = ((a & 127) == 127) & ((b & 127) == 127)      # the sign of a NaN says nothing
        assert np.array_equal(a[~nan], b[~nan]), x
    assert np.array_equal(got["scale"], want["scale"], equal_nan=True), "scale"
    assert np.array_equal(got["kmean"], want["kmean"], equal_nan=True), "kmean"


def make_batch(rng, seqs, page, pages, spare=1):
    """seqs: [(tokens held, new)].  Pages in random order; returns int32 (table, lens, cu)."""
    need = [-(-h // page) for h, _ in seqs]
    assert sum(need) <= pages
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((len(seqs), max(max(need), 1) + spare), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    lens = np.array([h for h, _ in seqs], dtype=np.int32)
    cu = np.concatenate([[0], np.cumsum([n for _, n in seqs])]).astype(np.int32)
    return table, lens, cu


def gpu_batch(batch, max_new, max_len=None):
    from paper_2605_15684_amd import cache
    return cache.Batch(*(torch.from_numpy(x.copy()).to("cuda") for x in batch), max_new, max_len)


def rounded(rng, shape, dtype, scale=1.0):
    """Normal values that `dtype` holds exactly: (torch tensor, float64 array)."""
    t = (torch.from_numpy(rng.standard_normal(shape)) * scale).to(dtype)
    return t, t.double().numpy()
