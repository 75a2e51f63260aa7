"""The paged 8-bit key/value cache and the attention that reads it: the calls whose time counts.

Kinds:
  append   new keys and values quantised into the pages of a cache (e4m3, one power-of-two scale per page and head)
  attend   attention of new tokens over everything their sequences hold in the cache
  sparse   block selection for each new token (pooled keys, top-k), then attention over the selected pages
  fork     one turn of a search: rows released, others forked into them, room made for the next token
  compact  live pages moved to the low end of the pool, the page table rewritten

A cache is four tensors: k and v [layers, pages, kv_heads, page * D] in e4m3, scale fp32 [layers, pages, kv_heads, 2]
(K's, V's) and kmean bf16 [layers, pages, kv_heads, D], the mean of the keys of each complete page.  The codes of a
page lie in the order of the matrix instructions' operands, 16 tokens after 16 tokens (_k_order, _v_order).  table int32 [seqs, max_pages] names the pages of each sequence in order (-1: none), lens
int32 [seqs] the tokens it holds with this call's, cu int32 [seqs + 1] where its new tokens lie in the packed arrays.

Sequences of a ragged case hold 50 to 100 % of `length`, bring 25 to 100 % of `new`, and every fifth one is idle.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_E4M3 = torch.float8_e4m3fn
_MIN_EXP = -64            # smallest exponent of a page's scale


def _case(name, kind, seqs, new, length, heads, kv_heads, d, page, dtype="bf16", ragged=False, causal=True, keep=0,
          layers=1):
    c = dict(kind=kind, seqs=seqs, new=new, length=length, heads=heads, kv_heads=kv_heads, d=d, page=page, dtype=dtype,
             ragged=ragged, causal=causal, keep=keep, layers=layers)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One token of each of eight sequences enters the cache: every layer of every generation step makes this call.
        _case("append_step", "append", 8, 1, 4096, 16, 4, 128, 64, ragged=True),
        # Four prompts at once.
        _case("append_prompts", "append", 4, 8192, 8192, 24, 8, 128, 64, ragged=True),
        # Full precision, small pages, a 77-token prompt behind what is there, one kv head per query head.
        _case("append_text77_f32", "append", 2, 77, 1101, 16, 16, 64, 16, dtype="f32"),
        # The smallest attention call: one token of one sequence.
        _case("attend_step1", "attend", 1, 1, 4096, 16, 4, 64, 64),
        # A full serving batch, one token each.
        _case("attend_step64", "attend", 64, 1, 16384, 16, 4, 128, 64, ragged=True),
        # Full precision, four drafted tokens each, small pages, three query heads to a kv head.
        _case("attend_draft4_f32", "attend", 16, 4, 2999, 24, 8, 128, 16, dtype="f32", ragged=True),
        # A 64x64-token image generated as one chunk behind three others: it sees all of itself.
        _case("attend_chunk4096", "attend", 1, 4096, 16384, 16, 4, 128, 64, causal=False),
        # The batch above, each token reading 32 pages of up to 256.
        _case("sparse_step64", "sparse", 64, 1, 16384, 16, 4, 128, 64, ragged=True, keep=32),
        # One sequence, very long.
        _case("sparse_long", "sparse", 1, 1, 262144, 16, 4, 128, 64, keep=64),
        # A chunk of 1024 tokens, each with pages of its own.
        _case("sparse_chunk1024", "sparse", 1, 1024, 12288, 24, 8, 64, 32, keep=20),
        # A search over 16 sequences in 24 layers: half the rows are dropped and forked anew from the others.
        _case("fork_24layers", "fork", 16, 1, 2029, 16, 4, 64, 64, ragged=True, layers=24),
        # A pool of 24 layers after half of its sequences have left.
        _case("compact_24layers", "compact", 32, 1, 1024, 16, 4, 64, 64, ragged=True, layers=24),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ranges: every kind, page size, type and head layout, odd lengths."""
    while True:
        kind = rng.choice(["append", "append", "attend", "attend", "attend", "sparse", "sparse", "sparse", "fork", "compact"])
        kv, d, page = _log_int(rng, 1, 16), rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 64])
        heads = kv * rng.choice([1, 2, 3, 4, 4, 6, 8, 16])
        seqs, keep, layers = _log_int(rng, 1, 64), 0, 1
        new = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 4096)])
        length = new + rng.choice([rng.randint(0, 40), _log_int(rng, 64, 16384), _log_int(rng, 64, 262144 if seqs == 1 else 16384)])
        if kind in ("fork", "compact"):
            layers, new, seqs, length = rng.randint(1, 24), 1, max(4, seqs), min(length, 4096)
        if kind == "sparse":
            keep = _log_int(rng, 4, 64)
        c = _case("", kind, seqs, new, length, heads, kv, d, page, rng.choice(["bf16", "bf16", "f32"]),
                  rng.random() < 0.7, rng.random() < 0.75, keep, layers)
        held = layers * seqs * length * kv * d
        if heads > 64 or held > 4 << 27 or seqs * new * heads * d > 1 << 25 or seqs * heads * new * length > 1 << 29:
            continue
        return c


# ---- the sequences of a case ------------------------------------------------------------------------------------

def _sequences(c):
    """[(tokens held after the call, new ones among them)] of each sequence: by the case alone."""
    out = []
    for s in range(c["seqs"]):
        held, new = c["length"], c["new"]
        if c["ragged"]:
            held = round(held * (0.5 + 0.5 * ((s + 1) * 0.6180339887 % 1)))
            new = max(1, round(new * (0.25 + 0.75 * ((s + 1) * 0.7548776662 % 1))))
            if s % 5 == 4:
                new = 0
        out.append((max(held, new), new))
    return out


def _children(c):
    """Rows of a fork case that are dropped and forked into from the row before them."""
    return list(range(1, c["seqs"], 2))


def _exponent(amax):
    """Smallest e >= _MIN_EXP with amax <= 448 * 2^e (448 = 1.75 * 2^8, the largest e4m3)."""
    m, x = torch.frexp(amax)                                  # amax = 2 m * 2^(x - 1), 2 m in [1, 2)
    e = torch.where(2 * m <= 1.75, x - 9, x - 8)
    return torch.where(amax > 0, e, _MIN_EXP).clamp(min=_MIN_EXP).to(torch.int32)


def _pow2(e):
    """2^e exactly, e in -126 .. 127."""
    return ((e.to(torch.int32).clamp(min=-126) + 127) << 23).view(torch.float32)


def _k_order(x):
    """[..., page, D] as a page keeps it: [16 tokens][64 channels][16 of them][token][channel]."""
    x = x.unflatten(-2, (-1, 16)).unflatten(-1, (-1, 4, 16))
    return x.movedim(-4, -2).flatten(-5)


def _k_rows(x, d):
    x = x.unflatten(-1, (-1, d // 64, 4, 16, 16)).movedim(-2, -4)
    return x.flatten(-3).flatten(-3, -2)


def _v_order(x):
    """[..., page, D] as a page keeps it: [16 tokens][64 channels][4 of the tokens][16 channels][4 such][token]."""
    x = x.unflatten(-2, (-1, 4, 4)).unflatten(-1, (-1, 4, 16))
    n = x.dim()
    return x.permute(*range(n - 5), n - 3, n - 5, n - 1, n - 2, n - 4).flatten(-6)


def _v_rows(x, d):
    x = x.unflatten(-1, (-1, d // 64, 4, 16, 4, 4))
    n = x.dim()
    return x.permute(*range(n - 5), n - 4, n - 1, n - 5, n - 2, n - 3).flatten(-3).flatten(-4, -2)


def _make_pool(c, pages, g):
    dev = "cuda"
    shape = (c["layers"], pages, c["kv_heads"])
    rows = (pages, c["kv_heads"], c["page"], c["d"])
    pool = {"k": torch.empty(shape + (c["page"] * c["d"],), dtype=_E4M3, device=dev),
            "v": torch.empty(shape + (c["page"] * c["d"],), dtype=_E4M3, device=dev),
            "scale": torch.empty(shape + (2,), dtype=torch.float32, device=dev),
            "kmean": torch.empty(shape + (c["d"],), dtype=torch.bfloat16, device=dev)}
    for layer in range(c["layers"]):
        for i, name in enumerate(("k", "v")):
            x = torch.randn(rows, generator=g, device=dev)
            x *= 0.5
            if name == "k":      # pages differ in where their keys point, as the topics of a text do
                x += 0.5 * torch.randn(x.shape[:2] + (1, c["d"]), generator=g, device=dev)
            s = _pow2(_exponent(x.abs().amax((-1, -2))))
            pool["scale"][layer, ..., i] = s
            x = (x / s[..., None, None]).to(_E4M3)
            pool[name][layer] = _k_order(x) if name == "k" else _v_order(x)
            if name == "k":
                pool["kmean"][layer] = (x.float().sum(-2) * (s / c["page"])[..., None]).to(torch.bfloat16)
    return pool


def prepare(case, seed):
    c = case
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    seqs = _sequences(c)
    need = [-(-held // c["page"]) for held, _ in seqs]
    max_pages = max(need) + 1
    pages = sum(need) + c["seqs"] + 3
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32).cpu()
    table = torch.full((c["seqs"], max_pages), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    cu = [0]
    for _, n in seqs:
        cu.append(cu[-1] + n)
    st = {"case": c, **_make_pool(c, pages, g), "table": table.to(dev), "rows": cu[-1],
          "lens": torch.tensor([h for h, _ in seqs], dtype=torch.int32, device=dev),
          "cu": torch.tensor(cu, dtype=torch.int32, device=dev), "max_new": max(n for _, n in seqs),
          "max_len": max(h for h, _ in seqs)}
    dt, rows = _DT[c["dtype"]], cu[-1]
    if c["kind"] == "append":
        # as a projection leaves them, one row in a hundred far larger
        kv = torch.randn((rows, 2, c["kv_heads"], c["d"]), generator=g, device=dev) * 0.5
        kv = torch.where(torch.rand((rows, 1, 1, 1), generator=g, device=dev) < 0.01, 8 * kv, kv).to(dt)
        st["new_k"], st["new_v"] = kv[:, 0], kv[:, 1]
    elif c["kind"] in ("attend", "sparse"):
        st["q"] = torch.randn((rows, c["heads"], c["d"]), generator=g, device=dev).to(dt)
    else:
        if c["kind"] == "compact":     # every second sequence has left
            st["table"][1::2] = -1
        refs = torch.zeros(pages, dtype=torch.int32)
        host = st["table"].cpu()
        refs[host[host >= 0].long()] = 1
        st["refs"] = refs.to(dev)
        kids = _children(c)
        st["dst"] = torch.tensor(kids, dtype=torch.int32, device=dev)
        st["src"] = st["dst"] - 1
    return st


# ---- the plain forms --------------------------------------------------------------------------------------------

def _rows_of(st):
    """Packed rows as [seqs, max_new]: the row's number and whether there is one."""
    n = st["cu"][1:] - st["cu"][:-1]
    i = torch.arange(st["max_new"], device=n.device)
    there = i < n[:, None]
    return torch.where(there, st["cu"][:-1, None] + i, 0).long(), there, n.long()


def _plain_append(st):
    c = st["case"]
    page = c["page"]
    rows, there, n = _rows_of(st)
    held = st["lens"].long()
    start = held - n
    first = start // page
    lp = first[:, None] + torch.arange((st["max_new"] + 2 * page - 2) // page, device=n.device)    # [S, P] pages touched
    touched = (n[:, None] > 0) & (lp * page < held[:, None])
    phys = torch.gather(st["table"].long(), 1, lp.clamp(max=st["table"].shape[1] - 1))
    seq, slot = touched.nonzero(as_tuple=True)
    lp, phys = lp[seq, slot], phys[seq, slot]                                                       # [T]
    pos = lp[:, None] * page + torch.arange(page, device=n.device)                                  # [T, page]
    is_new = (pos >= start[seq, None]) & (pos < held[seq, None])
    is_old = pos < start[seq, None]
    row = torch.where(is_new, st["cu"][seq, None].long() + pos - start[seq, None], 0)
    for i, (name, x) in enumerate((("k", st["new_k"]), ("v", st["new_v"]))):
        x = x.float()[row].transpose(1, 2)                                                          # [T, H, page, D]
        new = is_new[:, None, :, None]
        e = _exponent(torch.where(new, x, 0).abs().amax((-1, -2)))                                  # [T, H]
        before = torch.frexp(st["scale"][0, phys, :, i])[1] - 1
        e = torch.where(is_old.any(1)[:, None], torch.maximum(e, before), e)
        codes = _k_rows(st[name][0, phys], c["d"]) if name == "k" else _v_rows(st[name][0, phys], c["d"])
        old = (codes.float() * _pow2((before - e).clamp(max=0))[..., None, None]).to(_E4M3)
        out = torch.where(is_old[:, None, :, None], old.float(), codes.float())
        out = torch.where(new, (x * _pow2(-e)[..., None, None]).to(_E4M3).float(), out).to(_E4M3)
        st[name][0, phys] = _k_order(out) if name == "k" else _v_order(out)
        st["scale"][0, phys, :, i] = _pow2(e)
        if name == "k":
            full = (lp + 1) * page <= held[seq]
            mean = out.float().sum(-2) * (_pow2(e) / page)[..., None]
            st["kmean"][0, phys[full]] = mean[full].to(torch.bfloat16)
    return {x: st[x] for x in ("k", "v", "scale", "kmean")}


def _limits(st):
    """[seqs, max_new] keys each new token sees."""
    rows, there, n = _rows_of(st)
    held = st["lens"].long()[:, None]
    i = torch.arange(st["max_new"], device=held.device)
    return torch.where(there, held - n[:, None] + i + 1 if st["case"]["causal"] else held, 0)


def _plain_attend(st, lists=None):
    c = st["case"]
    d, page, kv = c["d"], c["page"], c["kv_heads"]
    rows, there, n = _rows_of(st)
    table = st["table"].long().clamp(min=0)
    scale = st["scale"][0][table]                                                                   # [S, P, H, 2]
    k = (_k_rows(st["k"][0][table], d).float() * scale[..., 0, None, None]).transpose(1, 2).reshape(len(n), kv, -1, d)
    v = (_v_rows(st["v"][0][table], d).float() * scale[..., 1, None, None]).transpose(1, 2).reshape(len(n), kv, -1, d)
    grp = c["heads"] // kv
    q = st["q"].float()[rows].view(len(n), -1, kv, grp, d).permute(0, 2, 1, 3, 4).reshape(len(n), kv, -1, d)
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(d)
    s = s.view(len(n), kv, -1, grp, s.shape[-1])
    sees = torch.arange(s.shape[-1], device=s.device) < _limits(st)[..., None]                      # [S, new, L]
    if lists is None:
        sees = sees[:, None, :, None]
    else:
        at = lists[rows].long()                                                                     # [S, new, H, 1+keep]
        kept = torch.zeros(at.shape[:3] + (table.shape[1] + 1,), dtype=torch.bool, device=s.device)
        kept = kept.scatter(-1, torch.where(at[..., 1:] < 0, table.shape[1], at[..., 1:]), True)[..., :-1]
        kept = kept.repeat_interleave(page, -1)
        sees = (sees[:, :, None] & kept).transpose(1, 2)[:, :, :, None]
    s = s.masked_fill(~sees, -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(len(n), kv, -1, p.shape[-1]), v).view(len(n), kv, -1, grp, d)
    o = o.permute(0, 2, 1, 3, 4).reshape(len(n), -1, c["heads"], d)
    out = torch.empty((st["rows"], c["heads"], d), dtype=st["q"].dtype, device=s.device)
    out[rows[there]] = o[there].to(out.dtype)
    return out


def _plain_select(st):
    c = st["case"]
    d, page, kv, keep = c["d"], c["page"], c["kv_heads"], c["keep"]
    rows, there, n = _rows_of(st)
    q = st["q"].double()[rows].view(len(n), -1, kv, c["heads"] // kv, d).sum(3).transpose(1, 2)     # [S, H, new, D]
    mean = st["kmean"][0][st["table"].long().clamp(min=0)].double().transpose(1, 2)                 # [S, H, P, D]
    score = torch.matmul(q, mean.transpose(-1, -2))
    last = (_limits(st) - 1).div(page, rounding_mode="floor")[:, None, :, None]                     # the token's own page
    j = torch.arange(score.shape[-1], device=score.device)
    score = torch.where((j < 1) | (j == last), math.inf, score)
    score = torch.where(j <= last, score, -math.inf)
    top = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :keep]
    top = torch.where(top <= last, top, score.shape[-1]).sort(-1)[0]
    count = (last + 1).clamp(max=keep)
    if top.shape[-1] < keep:
        top = torch.cat([top, torch.full(top.shape[:-1] + (keep - top.shape[-1],), score.shape[-1], device=top.device)], -1)
    ids = torch.where(top < score.shape[-1], top, -1)
    full = torch.cat([count.expand(ids.shape[:-1] + (1,)), ids], -1).transpose(1, 2)
    out = torch.empty((st["rows"], kv, 1 + keep), dtype=torch.int32, device=full.device)
    out[rows[there]] = full[there].to(torch.int32)
    return out


def _plain_fork(st):
    """Release the dst rows, fork the src rows into them, then give every sequence room for one more token."""
    c = st["case"]
    page, pages = c["page"], st["refs"].numel()
    table, lens, refs, src, dst = st["table"], st["lens"], st["refs"], st["src"].long(), st["dst"].long()
    gone = table[dst]
    refs -= torch.bincount(gone[gone >= 0].long(), minlength=pages).to(torch.int32)
    table[dst] = -1
    lens[dst] = 0
    held = lens[src].long()
    i = torch.arange(table.shape[1], device=held.device)
    rows = torch.where(i < (held // page)[:, None], table[src], -1)
    refs += torch.bincount(rows[rows >= 0].long(), minlength=pages).to(torch.int32)
    part = held % page != 0
    free = torch.sort((refs != 0).to(torch.int32), stable=True)[1][: int(part.sum())]
    old = table[src[part], held[part] // page].long()
    refs[free] = 1
    for x in ("k", "v", "scale", "kmean"):
        st[x][:, free] = st[x][:, old]
    table[dst] = rows
    table[dst[part], held[part] // page] = free.to(torch.int32)
    lens[dst] = lens[src]
    then = lens + (lens > 0)
    lacks = (i < ((then + page - 1) // page)[:, None]) & (table < 0)
    free = torch.sort((refs != 0).to(torch.int32), stable=True)[1][: int(lacks.sum())]
    refs[free] = 1
    table[lacks] = free.to(torch.int32)
    return {x: st[x] for x in ("table", "lens", "refs", "k", "v", "scale", "kmean")}


def _plain_compact(st):
    refs, pages = st["refs"], st["refs"].numel()
    live = refs > 0
    count = live.sum()
    i = torch.arange(pages, device=refs.device)
    src, dst = (live & (i >= count)).nonzero()[:, 0], (~live & (i < count)).nonzero()[:, 0]
    for x in ("k", "v", "scale", "kmean"):
        st[x][:, dst] = st[x][:, src]
    to = i.scatter(0, src, dst).to(torch.int32)
    new = refs.scatter(0, dst, refs[src]).scatter(0, src, 0)
    table = torch.where(st["table"] >= 0, to[st["table"].long().clamp(min=0)], st["table"])
    return {"table": table, "refs": new, "live": count.to(torch.int32), **{x: st[x] for x in ("k", "v", "scale", "kmean")}}


def _own(st):
    from paper_2605_15684_amd import cache
    c = st["case"]
    pool = cache.PagedCache(st["k"], st["v"], st["scale"], st["kmean"])
    state = {x: st[x] for x in ("k", "v", "scale", "kmean")}
    if c["kind"] == "fork":
        cache.release(pool, st["table"], st["lens"], st["refs"], st["dst"])
        cache.fork(pool, st["table"], st["lens"], st["refs"], st["src"], st["dst"])
        cache.reserve(pool, st["table"], st["lens"] + (st["lens"] > 0), st["refs"])
        return {"table": st["table"], "lens": st["lens"], "refs": st["refs"], **state}
    if c["kind"] == "compact":
        table, refs, info = cache.compact(pool, st["table"], st["refs"])
        return {"table": table, "refs": refs, "live": info[0], **state}
    batch = cache.Batch(st["table"], st["lens"], st["cu"], st["max_new"], st["max_len"])
    if c["kind"] == "append":
        cache.append(pool, 0, batch, st["new_k"], st["new_v"])
        return state
    if c["kind"] == "attend":
        return cache.attend(pool, 0, batch, st["q"], causal=c["causal"])
    lists = cache.select(pool, 0, batch, st["q"], keep=c["keep"], causal=c["causal"])
    return lists, cache.attend(pool, 0, batch, st["q"], lists=lists, causal=c["causal"])


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "append":
        return _plain_append(state)
    if kind == "attend":
        return _plain_attend(state)
    if kind == "sparse":
        lists = _plain_select(state)
        return lists, _plain_attend(state, lists)
    return _plain_fork(state) if kind == "fork" else _plain_compact(state)


def work(case):
    c = case
    seqs, size, page, kv = _sequences(c), _BYTES[c["dtype"]], c["page"], c["kv_heads"]
    rows = sum(n for _, n in seqs)
    payload = c["layers"] * kv * (2 * page * c["d"] + 8 + 2 * c["d"])       # one page, every layer
    if c["kind"] == "append":
        touched = sum(-(-h // page) - (h - n) // page for h, n in seqs if n)
        return {"bytes": rows * kv * c["d"] * 2 * (size + 1) + touched * kv * 8, "flops": 0}
    if c["kind"] == "fork":
        kids = _children(c)
        entries = sum(-(-seqs[s - 1][0] // page) for s in kids)
        return {"bytes": 2 * payload * sum(seqs[s - 1][0] % page != 0 for s in kids) + 12 * entries, "flops": 0}
    if c["kind"] == "compact":
        held = [-(-h // page) for h, _ in seqs]
        live, total = sum(held[::2]), sum(held) + c["seqs"] + 3
        moved = live * (total - live) / total                                # of pages in random places
        return {"bytes": 2 * payload * moved + 8 * total + 8 * sum(held), "flops": 0}
    io, pairs, keys, pooled = 2 * rows * c["heads"] * c["d"] * size, 0, 0, 0
    for h, n in seqs:
        if not n:
            continue
        sees = [h - n + i + 1 if c["causal"] else h for i in range(n)]
        if c["kind"] == "sparse":
            pairs += sum(min(x, c["keep"] * page) for x in sees)
            keys += min(h, n * c["keep"] * page)
            pooled += h // page
        else:
            pairs += sum(sees)
            keys += h
    lists = rows * kv * (1 + c["keep"]) * 4 if c["kind"] == "sparse" else 0
    return {"bytes": io + keys * kv * (2 * c["d"] + 8 / page) + pooled * kv * 2 * c["d"] + lists,
            "flops": 4 * c["d"] * c["heads"] * pairs}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _e4m3_of(x):
    """Nearest e4m3 value (ties to even) of float64 values of at most 448: a multiple of 2^(exponent - 3), at least 2^-9."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _places(page, d):
    """[page, D] the byte of a page that holds token t's channel ch, of K and of V."""
    t, ch = torch.arange(page, device="cuda")[:, None], torch.arange(d, device="cuda")
    block = (t // 16) * 16 * d + (ch // 64) * 1024
    k = block + (ch % 64 // 16) * 256 + (t % 16) * 16 + ch % 16
    return k, block + (t % 16 // 4) * 256 + (ch % 16) * 16 + (ch % 64 // 16) * 4 + t % 4


def _exact_append(c, st):
    page = c["page"]
    at = 0
    kat, vat = _places(page, c["d"])
    k, v, scale, mean = (st[x].double() for x in ("k", "v", "scale", "kmean"))
    for s, (held, n) in enumerate(_sequences(c)):
        start = held - n
        for lp in range(start // page, -(-held // page) if n else 0):
            phys = int(st["table"][s, lp])
            a, b = max(start, lp * page), min(held, (lp + 1) * page)
            for codes, where, i, x in ((k[0, phys], kat, 0, st["new_k"]), (v[0, phys], vat, 1, st["new_v"])):
                pool = codes[:, where]                                                 # [H, page, D]
                new = x[at + a - start:at + b - start].double().transpose(0, 1)        # [H, tokens, D]
                top = new.abs().amax((1, 2)).clamp(min=2.0 ** -200)
                e = torch.ceil(torch.log2(top / 448)).clamp(min=_MIN_EXP)
                e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
                e = torch.where((top <= 448 * torch.exp2(e - 1)) & (e > _MIN_EXP), e - 1, e)
                if a > lp * page:
                    was = scale[0, phys, :, i]
                    e = torch.maximum(e, torch.round(torch.log2(was)))
                    old = pool[:, :a - lp * page]
                    pool[:, :a - lp * page] = _e4m3_of(old * (was / torch.exp2(e))[:, None, None])
                scale[0, phys, :, i] = torch.exp2(e)
                pool[:, a - lp * page:b - lp * page] = _e4m3_of(new / torch.exp2(e)[:, None, None])
                codes[:, where] = pool
                if i == 0 and held >= (lp + 1) * page:
                    mean[0, phys] = pool.mean(1) * torch.exp2(e)[:, None]
        at += n
    return {"k": k, "v": v, "scale": scale, "kmean": mean}


def _exact_lists(c, st, s, held, n, q):
    """[n, H, P] which pages each token reads: the rank of every page counted from the scores."""
    page, kv = c["page"], c["kv_heads"]
    dev = q.device
    ids = st["table"][s, :-(-held // page)].long()
    scores = torch.einsum("nhgd,phd->nhp", q, st["kmean"][0, ids].double())
    seen = torch.arange(held - n + 1, held + 1, device=dev) if c["causal"] else torch.full((n,), held, device=dev)
    lastp = (seen - 1) // page
    j = torch.arange(len(ids), device=dev)
    kept = torch.empty(scores.shape, dtype=torch.bool, device=dev)
    for i in range(n):
        x = scores[i, :, :int(lastp[i]) + 1].clone()
        x[:, 0] = x[:, -1] = math.inf
        m = x.shape[1]
        kept[i] = False
        if m <= c["keep"]:
            kept[i, :, :m] = True
            continue
        bar = torch.topk(x, c["keep"], dim=1)[0][:, -1:]
        above = x > bar
        level = x == bar
        kept[i, :, :m] = above | (level & (level.cumsum(1) <= c["keep"] - above.sum(1, keepdim=True)))
    return kept


def exact(case, seed):
    c = case
    seqs = _sequences(c)
    if c["kind"] in ("fork", "compact"):
        return None                                            # nothing is computed: bytes and numbers of pages
    st = prepare(case, seed)
    if c["kind"] == "append":
        if sum(-(-n // c["page"]) + 1 for _, n in seqs) > 8000:
            return None
        return _exact_append(c, st)
    if c["kind"] == "sparse" and sum(n for _, n in seqs) > 4096:
        return None
    page, kv, d = c["page"], c["kv_heads"], c["d"]
    grp = c["heads"] // kv
    kat, vat = _places(page, d)
    out = torch.empty((st["rows"], c["heads"], d), dtype=torch.float64, device="cuda")
    at = 0
    for s, (held, n) in enumerate(seqs):
        if not n:
            continue
        ids = st["table"][s, :-(-held // page)].long()
        q = st["q"][at:at + n].double().view(n, kv, grp, d)
        j = torch.arange(len(ids) * page, device=q.device)
        seen = torch.arange(held - n + 1, held + 1, device=q.device) if c["causal"] else torch.full((n,), held, device=q.device)
        sees = (j < seen[:, None])[:, None].expand(n, kv, -1)
        if c["kind"] == "sparse":
            sees = sees & _exact_lists(c, st, s, held, n, q).repeat_interleave(page, -1)
        for h in range(kv):
            k = st["k"][0, ids, h].double()[:, kat] * st["scale"][0, ids, h, 0].double()[:, None, None]
            v = st["v"][0, ids, h].double()[:, vat] * st["scale"][0, ids, h, 1].double()[:, None, None]
            k, v = k.reshape(-1, d), v.reshape(-1, d)
            for g in range(grp):
                w = (q[:, h, g] @ k.T) * d ** -0.5
                w = torch.softmax(torch.where(sees[:, h], w, -math.inf), -1)
                out[at:at + n, h * grp + g] = w @ v
        at += n
    return out if c["kind"] == "attend" else (None, out)
