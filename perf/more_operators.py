"""Positions of several axes, attention that sees a window and the first tokens, attention over a shared prefix: the
calls whose time counts.

Kinds:
  rope    queries and keys turned by their tokens' positions on several axes (time, height, width); `inverse`: the
          gradients turned back
  window  attention of rows that are not cached, each over the last `window` tokens and the first `sinks`: output and
          log-sum-exp
  train   the same with its gradients: output, dq, dk, dv
  stream  attention of new tokens over a paged 8-bit cache, each over the last `window` tokens and the first `sinks`
  shared  attention of new tokens over a paged 8-bit cache whose sequences share the pages of a prefix, by groups

A turn of pair (a, b) by the angle phi = position[axis] * freq: (a cos phi - b sin phi, b cos phi + a sin phi).  With
sections (n0, n1, ...) the first n0 pairs go by axis 0 and so on, further pairs stay.  Spectrum "axis": pair i of a
section of n has freq theta^(-i/n); "shared": pair j of all D/2 has theta^(-j/(D/2)).  Pairs "adjacent": channels
(2j, 2j+1); "halves": (j, j + D/2).

The cache is that of perf/operators.py: e4m3 codes [layers, pages, kv_heads, page * D] in the order of the matrix
instructions' operands, scale fp32 [layers, pages, kv_heads, 2], kmean bf16; table, lens and cu as there.

Sequences of a ragged case hold 50 to 100 % of `length` (shared: of what they hold behind the prefix), bring 25 to
100 % of `new`, and every fifth one is idle; rows that are not cached are packed one sequence after another.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_E4M3 = torch.float8_e4m3fn


def _rope(name, rows, heads, kv_heads, d, dtype="bf16", packed=True, batch=1, grid=(1, 1), start=0, sections=(16, 24, 24),
          spectrum="axis", pairs="adjacent", theta=10000.0, inverse=False):
    return _named(name, dict(kind="rope", rows=rows, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, packed=packed,
                             batch=batch, grid_h=grid[0], grid_w=grid[1], start=start,
                             sections="-".join(str(n) for n in sections), spectrum=spectrum, pairs=pairs, theta=theta,
                             inverse=inverse))


def _rows(name, kind, seqs, length, heads, kv_heads, d, window, sinks, dtype="bf16", ragged=False):
    return _named(name, dict(kind=kind, seqs=seqs, length=length, heads=heads, kv_heads=kv_heads, d=d, window=window,
                             sinks=sinks, dtype=dtype, ragged=ragged))


def _cached(name, kind, seqs, new, length, heads, kv_heads, d, page, dtype="bf16", ragged=False, causal=True, window=0,
            sinks=0, groups=0, prefix=0):
    return _named(name, dict(kind=kind, seqs=seqs, new=new, length=length, heads=heads, kv_heads=kv_heads, d=d,
                             page=page, dtype=dtype, ragged=ragged, causal=causal, window=window, sinks=sinks,
                             groups=groups, prefix=prefix))


def _named(name, case):
    return {"name": name, **case} if name else case


def listed():
    return [
        # One new token of each of eight sequences, far into their streams: before every append of a generation step.
        _rope("rope_step8", 8, 16, 4, 128, start=100000),
        # 16 frames of 32x32 tokens of a video, as a prompt brings them; one spectrum over all axes.
        _rope("rope_video16384", 16384, 24, 8, 128, grid=(32, 32), spectrum="shared", pairs="halves", theta=1e6),
        # Gradients of four images of 64x64 tokens, full precision, two axes in use.
        _rope("rope_image_grad_f32", 4096, 16, 16, 64, dtype="f32", packed=False, batch=4, grid=(64, 64),
              sections=(0, 16, 16), inverse=True),
        # A prompt of 16384 tokens, forward alone.
        _rows("window_prompt16384", "window", 1, 16384, 16, 4, 128, 1024, 4),
        # Full precision, five packed sequences of odd lengths, a window that no tile divides.
        _rows("window_packed_f32", "window", 5, 1101, 6, 2, 64, 333, 5, dtype="f32", ragged=True),
        # The smallest training step.
        _rows("train_small", "train", 2, 200, 4, 4, 64, 64, 1),
        # One layer of a training step: two sequences of 8192.
        _rows("train_8192", "train", 2, 8192, 16, 4, 128, 2048, 16),
        # Packed documents, full precision, three query heads to a kv head.
        _rows("train_packed_f32", "train", 4, 2029, 6, 2, 128, 512, 4, dtype="f32", ragged=True),
        # One token of a long stream.
        _cached("stream_step1", "stream", 1, 1, 65536, 16, 4, 128, 64, window=1024, sinks=4),
        # A full serving batch, one token each.
        _cached("stream_step64", "stream", 64, 1, 16384, 16, 4, 128, 64, ragged=True, window=4096, sinks=64),
        # 64 samples of one prompt of 8192 tokens, one token each.
        _cached("shared_step64", "shared", 64, 1, 512, 16, 4, 128, 64, ragged=True, groups=1, prefix=8192),
        # Four prompts with four drafts each, full precision, small pages.
        _cached("shared_draft4_f32", "shared", 16, 4, 300, 24, 8, 64, 16, dtype="f32", ragged=True, groups=4,
                prefix=2992),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ranges: every kind, type, layout and head grouping, odd lengths."""
    kind = rng.choice(["rope", "rope", "window", "window", "train", "train", "train", "stream", "stream", "shared", "shared"])
    while True:
        dtype, d = rng.choice(["bf16", "bf16", "f32"]), rng.choice([64, 128, 128])
        kv, grp = _log_int(rng, 1, 16), rng.choice([1, 2, 3, 4, 4, 6, 8])
        heads = kv * grp
        if heads > 64:
            continue
        if kind == "rope":
            side = _log_int(rng, 1, 64)
            rows, batch, packed = _log_int(rng, 1, 16384), rng.choice([1, 1, 2, 4]), rng.random() < 0.5
            a, b = sorted((rng.randint(0, d // 2), rng.randint(0, d // 2)))
            sections = rng.choice([(a, b - a, d // 2 - b), (a, b - a), (d // 2,), (d // 8, 3 * d // 16, 3 * d // 16)])
            batch = 1 if packed else batch
            if rows * batch * (heads + kv) * d > 1 << 26:
                continue
            return _rope("", rows, heads, kv, d, dtype, packed, batch, (side, rng.randint(1, side)),
                         rng.choice([0, _log_int(rng, 1, 1 << 20)]), sections, rng.choice(["axis", "shared"]),
                         rng.choice(["adjacent", "halves"]), rng.choice([10000.0, 500000.0, 1e6]), rng.random() < 0.4)
        if kind in ("window", "train"):
            few = 8 if kind == "train" else 1        # one token alone has no gradient but rounding
            seqs, length = _log_int(rng, 1, 8), _log_int(rng, 2 * few, 16384)
            window, sinks = _log_int(rng, few, 4096), rng.choice([0, 1, 4, rng.randint(1, 200)])
            pairs = seqs * heads * length * min(length, 2 * window + sinks)
            if pairs > (1 << 30 if dtype == "bf16" else 1 << 27) or seqs * length * heads * d > 1 << 26:
                continue
            return _rows("", kind, seqs, length, heads, kv, d, window, sinks, dtype, rng.random() < 0.5)
        seqs, page = _log_int(rng, 1, 64), rng.choice([16, 32, 64, 64])
        new = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 1024)])
        c = dict(dtype=dtype, ragged=rng.random() < 0.7, causal=rng.random() < 0.8)
        if kind == "stream":
            length = new + rng.choice([rng.randint(0, 40), _log_int(rng, 64, 65536 if seqs < 4 else 16384)])
            c |= dict(window=_log_int(rng, 1, 4096), sinks=rng.choice([0, 1, 4, rng.randint(1, 200)]))
        else:
            groups = rng.randint(1, max(1, seqs // 2))
            length, prefix = new + _log_int(rng, 1, 1024), page * _log_int(rng, 1, 16384 // page)
            c |= dict(groups=groups, prefix=prefix)
        held = seqs * (length + c.get("prefix", 0))
        if held * kv * d > 1 << 28 or seqs * new * heads * d > 1 << 24 or held * new * heads > 1 << 28:
            continue
        return _cached("", kind, seqs, new, length, heads, kv, d, page, **c)


# ---- what a case holds --------------------------------------------------------------------------------------------

def _cached_sequences(c):
    """[(tokens held after the call, new ones among them)] of each sequence: by the case alone."""
    out = []
    for s in range(c["seqs"]):
        held, new = c["length"], c["new"]
        if c["ragged"]:
            held = round(held * (0.5 + 0.5 * ((s + 1) * 0.6180339887 % 1)))
            new = max(1, round(new * (0.25 + 0.75 * ((s + 1) * 0.7548776662 % 1))))
            if s % 5 == 4:
                new = 0
        out.append((c["prefix"] + max(held, new), new))
    return out


def _lengths(c):
    """Lengths of the sequences of rows."""
    if not c["ragged"]:
        return [c["length"]] * c["seqs"]
    return [0 if s % 5 == 4 else round(c["length"] * (0.5 + 0.5 * ((s + 1) * 0.6180339887 % 1))) for s in range(c["seqs"])]


def _group_of(c):
    """Group of each sequence: as even as they come, in order."""
    return [s * c["groups"] // c["seqs"] for s in range(c["seqs"])]


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
    shape, rows = (1, pages, c["kv_heads"]), (pages, c["kv_heads"], c["page"], c["d"])
    pool = {"k": torch.empty(shape + (c["page"] * c["d"],), dtype=_E4M3, device=dev),
            "v": torch.empty(shape + (c["page"] * c["d"],), dtype=_E4M3, device=dev),
            "scale": torch.empty(shape + (2,), dtype=torch.float32, device=dev),
            "kmean": torch.empty(shape + (c["d"],), dtype=torch.bfloat16, device=dev)}
    for i, name in enumerate(("k", "v")):
        x = torch.randn(rows, generator=g, device=dev) * 0.5
        if name == "k":      # pages differ in where their keys point, as the topics of a text do
            x += 0.5 * torch.randn(x.shape[:2] + (1, c["d"]), generator=g, device=dev)
        e = torch.ceil(torch.log2(x.abs().amax((-1, -2)) / 448))
        pool["scale"][0, ..., i] = torch.exp2(e)
        x = x * torch.exp2(-e)[..., None, None]
        pool[name][0] = (_k_order(x) if name == "k" else _v_order(x)).to(_E4M3)
        if name == "k":
            pool["kmean"][0] = (x.mean(-2) * torch.exp2(e)[..., None]).to(torch.bfloat16)
    return pool


def _prepare_cached(c, g):
    seqs, page, dev = _cached_sequences(c), c["page"], "cuda"
    shared = c["prefix"] // page
    need = [-(-held // page) - shared for held, _ in seqs]
    pages = sum(need) + c["groups"] * shared + 3
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32).cpu()
    table = torch.full((c["seqs"], max(need) + shared + 1), -1, dtype=torch.int32)
    at = c["groups"] * shared
    for s, n in enumerate(need):
        if shared:
            mine = _group_of(c)[s] * shared
            table[s, :shared] = order[mine:mine + shared]
        table[s, shared:shared + n] = order[at:at + n]
        at += n
    cu = [0]
    for _, n in seqs:
        cu.append(cu[-1] + n)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    st = {**_make_pool(c, pages, g), "table": table.to(dev), "rows": cu[-1], "lens": ints([h for h, _ in seqs]),
          "cu": ints(cu), "max_new": max(n for _, n in seqs), "max_len": max(h for h, _ in seqs)}
    if c["kind"] == "shared":
        group = _group_of(c)
        first = [group.index(x) for x in range(c["groups"])] + [c["seqs"]]
        st["first"], st["pages"] = ints(first), ints([shared] * c["groups"])
        st["group_seqs"] = max(b - a for a, b in zip(first, first[1:]))
    st["q"] = torch.randn((cu[-1], c["heads"], c["d"]), generator=g, device=dev).to(_DT[c["dtype"]])
    return st


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    st = {"case": c}
    dt, d = _DT[c["dtype"]], c["d"]
    randn = lambda *shape: torch.randn(shape, generator=g, device=dev).to(dt)
    if c["kind"] == "rope":
        sections = [int(n) for n in c["sections"].split("-")]
        i = torch.arange(c["rows"], device=dev)
        area = c["grid_h"] * c["grid_w"]
        at = (i // area + c["start"], i % area // c["grid_w"], i % c["grid_w"])     # (time, height, width)
        st["pos"] = torch.stack(at[:len(sections)], -1).to(torch.int32)
        for name, heads in (("q", c["heads"]), ("k", c["kv_heads"])):
            st[name] = randn(c["rows"], heads, d) if c["packed"] else randn(c["batch"], heads, c["rows"], d)
        st["sections"] = sections
        return st
    if c["kind"] in ("stream", "shared"):
        return st | _prepare_cached(c, g)
    lens = _lengths(c)
    st["lens"], st["max_len"] = lens, max(lens)
    for name, heads in (("q", c["heads"]), ("k", c["kv_heads"]), ("v", c["kv_heads"]), ("do", c["heads"])):
        if name == "do" and c["kind"] == "window":
            continue
        st[name] = randn(sum(lens), heads, d) if c["ragged"] else randn(c["seqs"], heads, c["length"], d)
    if c["ragged"]:
        st["cu"] = torch.tensor([sum(lens[:s]) for s in range(len(lens) + 1)], dtype=torch.int32, device=dev)
    return st


# ---- the plain forms --------------------------------------------------------------------------------------------

def _plain_rope(st):
    c, sections, half = st["case"], st["sections"], st["case"]["d"] // 2
    dev = st["pos"].device
    axis = torch.cat([torch.full((n,), a, device=dev) for a, n in enumerate(sections)])
    if c["spectrum"] == "axis":
        power = torch.cat([torch.arange(n, dtype=torch.float64, device=dev) / max(n, 1) for n in sections])
    else:
        power = torch.arange(len(axis), dtype=torch.float64, device=dev) / half
    phi = st["pos"].double()[:, axis] * c["theta"] ** -power                          # [rows, turned pairs]
    phi = torch.cat([phi, phi.new_zeros(phi.shape[0], half - phi.shape[1])], -1)
    cos, sin = torch.cos(phi).float(), torch.sin(phi).float()
    if c["inverse"]:
        sin = -sin
    if c["packed"]:
        cos, sin = cos[:, None], sin[:, None]
    out = []
    for x in (st["q"], st["k"]):
        y = x.float()
        a, b = (y[..., 0::2], y[..., 1::2]) if c["pairs"] == "adjacent" else (y[..., :half], y[..., half:])
        a, b = a * cos - b * sin, b * cos + a * sin
        y = torch.stack([a, b], -1).flatten(-2) if c["pairs"] == "adjacent" else torch.cat([a, b], -1)
        out.append(y.to(x.dtype))
    return tuple(out)


def _padded(st, x):
    """Rows as [seqs, heads, length, D] in fp32, zeros behind a sequence's end."""
    if "cu" not in st:
        return x.float()
    n = st["cu"][1:] - st["cu"][:-1]
    i = torch.arange(st["max_len"], device=x.device)
    there = i < n[:, None]
    rows = torch.where(there, st["cu"][:-1, None] + i, 0).long()
    return torch.where(there[..., None, None], x.float()[rows], 0).transpose(1, 2)


def _unpadded(st, x, dtype):
    """The other way, [heads, length] among them; values rounded to dtype."""
    if "cu" not in st:
        return x.to(dtype)
    n = st["cu"][1:] - st["cu"][:-1]
    seq, at = (torch.arange(x.shape[2], device=x.device) < n[:, None]).nonzero(as_tuple=True)
    x = x[seq, :, at].to(dtype)
    return x if x.dim() == 3 else x.transpose(0, 1).contiguous()


def _blocks(x, size):
    """[S, H, L, D] in blocks [S, H, n, size, D], zeros at the end."""
    x = torch.nn.functional.pad(x, (0, 0, 0, -x.shape[2] % size))
    return x.unflatten(2, (-1, size))


def _with_before(x):
    """Each block behind the one before it: [S, H, n, 2 size, D]."""
    before = torch.cat([torch.zeros_like(x[:, :, :1]), x[:, :, :-1]], 2)
    return torch.cat([before, x], 3)


def _plain_rows(st):
    c = st["case"]
    kv, grp, d = c["kv_heads"], c["heads"] // c["kv_heads"], c["d"]
    q, k, v = (_padded(st, st[x]) for x in ("q", "k", "v"))
    length = q.shape[2]
    size = min(c["window"], length)                 # blocks as long as the window: a token sees its block and the one before
    sinks = min(c["sinks"], length)
    kb, vb = (_with_before(_blocks(x, size)) for x in (k, v))
    n = kb.shape[2]
    group = lambda x: _blocks(x, size).unflatten(1, (kv, grp)).transpose(2, 3).flatten(3, 4)    # [S, KV, n, G size, D]
    ungroup = lambda x: x.unflatten(3, (grp, size)).transpose(2, 3).flatten(1, 2).flatten(2, 3)[:, :, :length]
    q = group(q)
    first = lambda x: x[:, :, None, :sinks].expand(-1, -1, n, -1, -1)
    keys, values = torch.cat([first(k), kb], 3), torch.cat([first(v), vb], 3)
    s = torch.matmul(q, keys.transpose(-1, -2)) / math.sqrt(d)
    i = torch.arange(n * size, device=q.device).view(n, 1, size, 1)
    at = (torch.arange(n, device=q.device)[:, None] - 1) * size + torch.arange(2 * size, device=q.device)
    near = (at >= 0)[:, None, None] & (at[:, None, None] <= i) & (at[:, None, None] > i - c["window"])
    early = (torch.arange(sinks, device=q.device) <= i - c["window"])
    sees = torch.cat([early, near], -1).expand(n, grp, size, -1).flatten(1, 2)
    s = s.masked_fill_(~sees, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    p = p / total
    o = torch.matmul(p, values)
    dt = st["q"].dtype
    if c["kind"] == "window":
        return _unpadded(st, ungroup(o), dt), _unpadded(st, ungroup(top + torch.log(total))[..., 0], torch.float32)
    do = group(_padded(st, st["do"]))
    ds = p * (torch.matmul(do, values.transpose(-1, -2)) - (do * o).sum(-1, keepdim=True)) / math.sqrt(d)
    dq = torch.matmul(ds, keys)

    def fold(x):                                     # gradients of `first` and of `_with_before`
        near = x[:, :, :, sinks + size:]
        near = near + torch.cat([x[:, :, 1:, sinks:sinks + size], torch.zeros_like(near[:, :, :1])], 2)
        near = near.flatten(2, 3)[:, :, :length]
        near[:, :, :sinks] += x[:, :, :, :sinks].sum(2)
        return near

    dk, dv = fold(torch.matmul(ds.transpose(-1, -2), q)), fold(torch.matmul(p.transpose(-1, -2), do))
    return tuple(_unpadded(st, x, dt) for x in (ungroup(o), ungroup(dq), dk, dv))


def _plain_cached(st):
    c = st["case"]
    d, kv, grp = c["d"], c["kv_heads"], c["heads"] // c["kv_heads"]
    n = (st["cu"][1:] - st["cu"][:-1]).long()
    i = torch.arange(st["max_new"], device=n.device)
    there = i < n[:, None]
    rows = torch.where(there, st["cu"][:-1, None] + i, 0).long()
    held = st["lens"].long()[:, None]
    at = torch.where(there, held - n[:, None] + i, 0)                                                 # positions
    limit = torch.where(there, at + 1 if c["causal"] else held, 0)
    table = st["table"].long().clamp(min=0)
    scale = st["scale"][0][table]                                                                   # [S, P, H, 2]
    k = (_k_rows(st["k"][0][table], d).float() * scale[..., 0, None, None]).transpose(1, 2).reshape(len(n), kv, -1, d)
    v = (_v_rows(st["v"][0][table], d).float() * scale[..., 1, None, None]).transpose(1, 2).reshape(len(n), kv, -1, d)
    q = st["q"].float()[rows].view(len(n), -1, kv, grp, d).permute(0, 2, 1, 3, 4).reshape(len(n), kv, -1, d)
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(d)
    s = s.view(len(n), kv, -1, grp, s.shape[-1])
    j = torch.arange(s.shape[-1], device=s.device)
    sees = j < limit[..., None]                                                                       # [S, new, L]
    if c["kind"] == "stream":
        sees = sees & ((j < c["sinks"]) | (j > at[..., None] - c["window"]))
    s = s.masked_fill_(~sees[:, None, :, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(len(n), kv, -1, p.shape[-1]), v).view(len(n), kv, -1, grp, d)
    o = o.permute(0, 2, 1, 3, 4).reshape(len(n), -1, c["heads"], d)
    out = torch.empty((st["rows"], c["heads"], d), dtype=st["q"].dtype, device=s.device)
    out[rows[there]] = o[there].to(out.dtype)
    return out


def _own(st):
    c = st["case"]
    if c["kind"] == "rope":
        from paper_2605_15684_amd import rope
        if "plan" not in st:                        # made once by a program
            st["plan"] = rope.plan(c["d"], st["sections"], theta=c["theta"], spectrum=c["spectrum"], pairs=c["pairs"])
        return rope.rotate(st["plan"], st["pos"], st["q"], st["k"], inverse=c["inverse"])
    if c["kind"] in ("window", "train"):
        from paper_2605_15684_amd import window
        sees = dict(window=c["window"], sinks=c["sinks"], cu=st.get("cu"), max_len=st["max_len"])
        o, lse = window.forward(st["q"], st["k"], st["v"], **sees)
        if c["kind"] == "window":
            return o, lse
        return (o,) + window.backward(st["q"], st["k"], st["v"], o, st["do"], lse, **sees)
    from paper_2605_15684_amd import cache
    if "pool" not in st:                            # made once by a program
        st["pool"] = cache.PagedCache(st["k"], st["v"], st["scale"], st["kmean"])
    batch = cache.Batch(st["table"], st["lens"], st["cu"], st["max_new"], st["max_len"])
    if c["kind"] == "stream":
        return cache.attend_window(st["pool"], 0, batch, st["q"], window=c["window"], sinks=c["sinks"],
                                   causal=c["causal"])
    prefix = cache.Prefix(st["first"], st["pages"], st["group_seqs"], c["prefix"])
    return cache.attend_shared(st["pool"], 0, batch, prefix, st["q"], causal=c["causal"])


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "rope":
        return _plain_rope(state)
    return _plain_rows(state) if kind in ("window", "train") else _plain_cached(state)


def _seen(at, window, sinks, limit):
    """Keys that the token at position `at` sees among the first `limit`."""
    low = max(at - window + 1, 0)
    return limit - low + min(sinks, low) if limit > low else min(sinks, limit)


def work(case):
    c = case
    size, d, heads, kv = _BYTES[c["dtype"]], c["d"], c["heads"], c["kv_heads"]
    if c["kind"] == "rope":
        axes = len(c["sections"].split("-"))
        values = c["batch"] * c["rows"] * (heads + kv) * d
        return {"bytes": 2 * values * size + 4 * axes * c["rows"], "flops": 3 * values}
    if c["kind"] in ("window", "train"):
        rows = sum(_lengths(c))
        pairs = heads * sum(_seen(i, c["window"], c["sinks"], i + 1) for n in _lengths(c) for i in range(n))
        if c["kind"] == "window":
            return {"bytes": rows * (2 * heads + 2 * kv) * d * size + 4 * rows * heads, "flops": 4 * d * pairs}
        return {"bytes": rows * (4 * heads + 4 * kv) * d * size, "flops": 14 * d * pairs}
    pairs, keys = 0, 0
    for h, n in _cached_sequences(c):
        if not n:
            continue
        if c["kind"] == "stream":
            pairs += sum(_seen(i, c["window"], c["sinks"], i + 1 if c["causal"] else h) for i in range(h - n, h))
            keys += _seen(h - n, c["window"], c["sinks"], h)
        else:
            pairs += sum(i + 1 if c["causal"] else h for i in range(h - n, h))
            keys += h - c["prefix"]
    rows = sum(n for _, n in _cached_sequences(c))
    keys += c["groups"] * c["prefix"]
    return {"bytes": 2 * rows * heads * d * size + keys * kv * (2 * d + 8 / c["page"]), "flops": 4 * d * heads * pairs}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_rope(c, st):
    half, base = c["d"] // 2, math.log(c["theta"])
    turns = []                                       # (pair, axis, frequency)
    pair = 0
    for axis, n in enumerate(st["sections"]):
        for i in range(n):
            turns.append((pair, axis, math.exp(-base * (i / n if c["spectrum"] == "axis" else pair / half))))
            pair += 1
    out = []
    for x in (st["q"], st["k"]):
        y = x.double().clone()
        for j, axis, f in turns:
            a, b = (2 * j, 2 * j + 1) if c["pairs"] == "adjacent" else (j, j + half)
            z = torch.complex(x[..., a].double(), x[..., b].double())
            phi = st["pos"][:, axis].double() * (-f if c["inverse"] else f)
            w = torch.complex(torch.cos(phi), torch.sin(phi))
            z = z * (w[:, None] if c["packed"] else w)
            y[..., a], y[..., b] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_rows(c, st):
    grp, step, dev = c["heads"] // c["kv_heads"], 512, "cuda"
    rows = lambda x: x if c["ragged"] else x.transpose(1, 2).flatten(0, 1)          # [rows, heads, D]
    q, k, v = (rows(st[x]).double() for x in ("q", "k", "v"))
    out = [torch.zeros_like(q)]
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=dev)
    train = c["kind"] == "train"
    if train:
        do = rows(st["do"]).double()
        out += [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]
    begin = 0
    for n in _lengths(c):
        for a in range(0, n, step):
            b = min(n, a + step)
            j = torch.arange(b, device=dev)
            j = j[(j < c["sinks"]) | (j > a - c["window"])]
            i = torch.arange(a, b, device=dev)[:, None]
            hidden = (j > i) | ((j >= c["sinks"]) & (j <= i - c["window"]))
            for h in range(c["heads"]):
                mine = [q[begin + a:begin + b, h], k[begin + j, h // grp], v[begin + j, h // grp]]
                mine = [x.detach().requires_grad_(train) for x in mine]
                s = (mine[0] @ mine[1].T * c["d"] ** -0.5).masked_fill(hidden, -math.inf)
                o = torch.softmax(s, -1) @ mine[2]
                out[0][begin + a:begin + b, h] = o.detach()
                lse[begin + a:begin + b, h] = torch.logsumexp(s.detach(), -1)
                if train:
                    gq, gk, gv = torch.autograd.grad(o, mine, do[begin + a:begin + b, h])
                    out[1][begin + a:begin + b, h] = gq
                    out[2][begin + j, h // grp] += gk
                    out[3][begin + j, h // grp] += gv
        begin += n
    if not c["ragged"]:
        out = [x.unflatten(0, (c["seqs"], -1)).transpose(1, 2) for x in out]
        lse = lse.unflatten(0, (c["seqs"], -1)).transpose(1, 2)
    else:
        lse = lse.T
    return tuple(out) if train else (out[0], lse)


def _places(page, d):
    """[page, D] the byte of a page that holds token t's channel ch, of K and of V."""
    t, ch = torch.arange(page, device="cuda")[:, None], torch.arange(d, device="cuda")
    block = (t // 16) * 16 * d + (ch // 64) * 1024
    k = block + (ch % 64 // 16) * 256 + (t % 16) * 16 + ch % 16
    return k, block + (t % 16 // 4) * 256 + (ch % 16) * 16 + (ch % 64 // 16) * 4 + t % 4


def _exact_cached(c, st):
    page, kv, d = c["page"], c["kv_heads"], c["d"]
    grp = c["heads"] // kv
    kat, vat = _places(page, d)
    out = torch.empty((st["rows"], c["heads"], d), dtype=torch.float64, device="cuda")
    at = 0
    for s, (held, n) in enumerate(_cached_sequences(c)):
        if not n:
            continue
        ids = st["table"][s, :-(-held // page)].long()
        j = torch.arange(len(ids) * page, device="cuda")
        i = torch.arange(held - n, held, device="cuda")[:, None]
        hidden = (j > i) if c["causal"] else (j >= held).expand(n, -1)
        if c["kind"] == "stream":
            hidden = hidden | ((j >= c["sinks"]) & (j <= i - c["window"]))
        for h in range(kv):
            k = st["k"][0, ids, h].double()[:, kat] * st["scale"][0, ids, h, 0].double()[:, None, None]
            v = st["v"][0, ids, h].double()[:, vat] * st["scale"][0, ids, h, 1].double()[:, None, None]
            q = st["q"][at:at + n, h * grp:(h + 1) * grp].double().transpose(0, 1)
            w = torch.softmax((q @ k.reshape(-1, d).T * d ** -0.5).masked_fill(hidden, -math.inf), -1)
            out[at:at + n, h * grp:(h + 1) * grp] = (w @ v.reshape(-1, d)).transpose(0, 1)
        at += n
    return out


def exact(case, seed):
    c = case
    if c["kind"] in ("window", "train") and c["heads"] * sum(-(-n // 512) for n in _lengths(c)) > 3000:
        return None
    st = prepare(c, seed)
    if c["kind"] == "rope":
        return _exact_rope(c, st)
    return _exact_rows(c, st) if c["kind"] in ("window", "train") else _exact_cached(c, st)
