"""Plain fp64 implementation of the paged 8-bit key/value cache (include/ssba_cache.h).

NumPy on the CPU, token by token and page by page; shares no code with the
GPU path.  A pool is a dict: k, v uint8 [layers, pages, kv_heads, page * D],
scale float32 [..., 2], kmean float32 (bf16 values) [..., D].  A batch is
(table, lens, cu) of int arrays.
"""
import numpy as np

MIN_EXP = -64


# ---- e4m3 -----------------------------------------------------------------

def _decode_table():
    out = np.zeros(256)
    for code in range(256):
        sign = -1.0 if code & 128 else 1.0
        exp, man = (code >> 3) & 15, code & 7
        if exp == 15 and man == 7:
            out[code] = np.nan
        elif exp == 0:
            out[code] = sign * man * 2.0 ** -9
        else:
            out[code] = sign * (1 + man / 8) * 2.0 ** (exp - 7)
    return out


E4M3 = _decode_table()


def e4m3(x):
    """Codes (uint8) of float64 values: nearest, ties to even, +-inf and anything above 448 as +-448."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    nan = np.isnan(x)
    a = np.where(nan, 0.0, a)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -6))), -6) - 3)
    r = np.rint(a / step) * step                       # np.rint: half to even
    exp = np.floor(np.log2(np.maximum(r, 2.0 ** -6)))
    normal = r >= 2.0 ** -6
    code = np.where(normal, (exp + 7) * 8 + (r / 2.0 ** exp - 1) * 8, r * 2.0 ** 9).astype(np.int64)
    code = np.where(nan, 127, code)
    return (code | np.where(np.signbit(x) & ~nan, 128, 0)).astype(np.uint8)


def exponent(amax):
    """Smallest e >= MIN_EXP with amax <= 448 * 2^e."""
    e = MIN_EXP
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def reach(s):
    """Smallest e >= MIN_EXP with s <= 2^e."""
    m, x = np.frexp(s)                                 # s = m 2^x, m in [1/2, 1)
    return max(int(x) - (m == 0.5), MIN_EXP)


def to_bf16(x):
    """float64 -> nearest bf16 (ties to even), as float32; the value must not need double rounding."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r)


# ---- order of the bytes of a page ------------------------------------------

def k_byte(t, c, d):
    return 16 * d * (t // 16) + 1024 * (c // 64) + 256 * (c % 64 // 16) + 16 * (t % 16) + c % 16


def v_byte(t, c, d):
    return 16 * d * (t // 16) + 1024 * (c // 64) + 256 * (t % 16 // 4) + 16 * (c % 16) + 4 * (c % 64 // 16) + t % 4


def orders(page, d):
    t, c = np.arange(page)[:, None], np.arange(d)[None, :]
    return k_byte(t, c, d), v_byte(t, c, d)


def rows_of(pool, layer, phys, head, which, page, d):
    """The keys (which 0) or values (1) of a page as float64 [page, D]."""
    codes = pool["kv"[which]][layer, phys, head][orders(page, d)[which]]
    return E4M3[codes] * np.float64(pool["scale"][layer, phys, head, which])


# ---- the calls ---------------------------------------------------------------

def sequences(batch, page, rows):
    """(begin, new, start, len) of each sequence, cut to the arrays as the header says; start: where the first new
    token is, by the length as it is given."""
    table, lens, cu = batch
    out = []
    for s in range(len(lens)):
        begin = min(max(int(cu[s]), 0), rows)
        end = max(min(int(cu[s + 1]), rows), begin)
        held = max(int(lens[s]), 0)
        out.append((begin, end - begin, held - (end - begin), min(held, table.shape[1] * page)))
    return out


def append(pool, layer, batch, k, v, page):
    """k, v float64 [rows, kv_heads, D]; updates pool."""
    table = batch[0]
    rows, heads, d = k.shape
    pages = pool["k"].shape[1]
    order = orders(page, d)
    for s, (begin, n, start, held) in enumerate(sequences(batch, page, rows)):
        if n == 0 or start < 0:
            continue
        for lp in range(start // page, (held - 1) // page + 1):
            phys = int(table[s, lp])
            if not 0 <= phys < pages:
                continue
            lo, hi = max(start, lp * page), min(held, (lp + 1) * page)
            for h in range(heads):
                for which, x in enumerate((k, v)):
                    new = x[begin + lo - start:begin + hi - start, h]
                    finite = np.abs(new[np.isfinite(new)])
                    e = exponent(finite.max() if finite.size else 0.0)
                    codes = pool["kv"[which]][layer, phys, h]
                    if lp * page < start:
                        was = float(pool["scale"][layer, phys, h, which])
                        e = max(e, min(reach(was), 120))
                        f = np.float32(was * 2.0 ** -e)
                        if f != 1:
                            at = order[which][:lo - lp * page]
                            codes[at] = e4m3(E4M3[codes[at]].astype(np.float32) * f)
                    codes[order[which][lo - lp * page:hi - lp * page]] = e4m3(new * 2.0 ** -e)
                    pool["scale"][layer, phys, h, which] = 2.0 ** e
                    if which == 0 and held >= (lp + 1) * page:
                        pool["kmean"][layer, phys, h] = to_bf16(E4M3[codes[order[0]]].sum(0) * 2.0 ** e / page)


def visible(start, held, tok, causal):
    return min(max(start + tok + 1, 0), held) if causal else held


def select(pool, layer, batch, q, page, keep, first=1, last=1, causal=True):
    """q float64 [rows, heads, D] -> int32 [rows, kv_heads, 1 + keep]; rows of no sequence are -7."""
    table = batch[0]
    rows, heads, d = q.shape
    pages, kv = pool["k"].shape[1:3]
    out = np.full((rows, kv, 1 + keep), -7, dtype=np.int32)
    for s, (begin, n, start, held) in enumerate(sequences(batch, page, rows)):
        for tok in range(n):
            sees = visible(start, held, tok, causal)
            total = (sees - 1) // page + 1 if sees > 0 else 0
            for h in range(kv):
                ids = list(range(total))
                if total > keep:
                    qs = np.zeros(d)
                    for g in range(heads // kv):
                        qs = qs + q[begin + tok, h * (heads // kv) + g]
                    middle = []
                    for j in range(first, total - last):
                        p = int(table[s, j])
                        score = -np.inf
                        rank = 0                                     # NaN, or not there: behind every number
                        if 0 <= p < pages:
                            score = float(np.dot(qs, pool["kmean"][layer, p, h].astype(np.float64)))
                            rank = 0 if np.isnan(score) else 1
                        middle.append((-rank, -score if rank else 0.0, j))
                    chosen = sorted(j for _, _, j in sorted(middle)[:keep - first - last])
                    ids = list(range(first)) + chosen + list(range(total - last, total))
                out[begin + tok, h] = [len(ids)] + ids + [-1] * (keep - len(ids))
    return out


def attend(pool, layer, batch, q, page, lists=None, causal=True, scale=None):
    """Returns (o, weight, spread): o float64 [rows, heads, D] with NaN rows where no sequence has one; weight =
    sum_j p_j |v_j| and spread = max_j scale sum |q k_j| over the visible keys, for error bounds."""
    table = batch[0]
    rows, heads, d = q.shape
    pages, kv = pool["k"].shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    o = np.full((rows, heads, d), np.nan)
    weight, spread = np.zeros((rows, heads, d)), np.zeros((rows, heads))
    for s, (begin, n, start, held) in enumerate(sequences(batch, page, rows)):
        for h in range(kv):
            known = {}

            def get(lp):
                if lp not in known:
                    p = int(table[s, lp])
                    known[lp] = None if not 0 <= p < pages else [rows_of(pool, layer, p, h, w, page, d) for w in (0, 1)]
                return known[lp]

            for tok in range(n):
                sees = visible(start, held, tok, causal)
                if lists is None:
                    use = range(-(-sees // page))
                else:
                    row = lists[begin + tok, h]
                    use = [int(x) for x in row[1:1 + min(max(int(row[0]), 0), lists.shape[2] - 1)]]
                ks, vs = [], []
                for lp in use:
                    if 0 <= lp < table.shape[1] and lp * page < sees and get(lp) is not None:
                        m = min(page, sees - lp * page)
                        ks.append(get(lp)[0][:m])
                        vs.append(get(lp)[1][:m])
                for g in range(heads // kv):
                    r, head = begin + tok, h * (heads // kv) + g
                    if not ks:
                        o[r, head] = 0.0
                        continue
                    kk, vv = np.concatenate(ks), np.concatenate(vs)
                    w = scale * (kk @ q[r, head])
                    p = np.exp(w - w.max())
                    p /= p.sum()
                    o[r, head] = p @ vv
                    weight[r, head] = p @ np.abs(vv)
                    spread[r, head] = abs(scale) * (np.abs(kk) @ np.abs(q[r, head])).max()
    return o, weight, spread


# ---- pages (table, lens, refs updated in place; payload through `pool` where given) ----

def _free(refs):
    return [p for p in range(len(refs)) if refs[p] == 0]


def reserve(table, lens, refs, page):
    free, got, short = _free(refs), 0, 0
    for s in range(len(lens)):
        for i in range(min(-(-max(int(lens[s]), 0) // page), table.shape[1])):
            if 0 <= table[s, i] < len(refs):
                continue
            if free:
                table[s, i] = free.pop(0)
                refs[table[s, i]] = 1
                got += 1
            else:
                short += 1
    return got, short


def _copy_page(pool, src, dst):
    for x in ("k", "v", "scale", "kmean"):
        pool[x][:, dst] = pool[x][:, src]


def fork(pool, table, lens, refs, src, dst, page):
    rows, most = table.shape
    sources = {int(x) for x in src if 0 <= x < rows}
    done, partial, cut = set(), [], 0
    for x, y in zip(src, dst):
        x, y = int(x), int(y)
        if not (0 <= x < rows and 0 <= y < rows):
            if 0 <= y < rows:
                done.add(y)
            continue
        if y in done or y in sources:
            continue
        done.add(y)
        held = min(max(int(lens[x]), 0), most * page)
        full = held // page
        table[y] = -1
        for i in range(full):
            if 0 <= table[x, i] < len(refs):
                table[y, i] = table[x, i]
                refs[table[x, i]] += 1
        lens[y] = held
        partial.append((x, y, full, held % page))
    free = _free(refs)
    for x, y, full, rest in partial:
        if rest and 0 <= table[x, full] < len(refs):
            if free:
                p = free.pop(0)
                refs[p] = 1
                table[y, full] = p
                _copy_page(pool, int(table[x, full]), p)
            else:
                lens[y] = full * page
                cut += 1
    return len(partial), cut


def release(table, lens, refs, rows):
    dropped = freed = 0
    done = set()
    for r in rows:
        r = int(r)
        if not 0 <= r < len(lens) or r in done:
            continue
        done.add(r)
        for i in range(table.shape[1]):
            p = int(table[r, i])
            if 0 <= p < len(refs):
                dropped += 1
                if refs[p] > 0:
                    refs[p] -= 1
                    freed += refs[p] == 0
            table[r, i] = -1
        lens[r] = 0
    return dropped, int(freed)


def compact(pool, table, refs):
    """Returns (table, refs, pages in use, pages moved)."""
    live = int((refs > 0).sum())
    to = np.arange(len(refs))
    movers = [p for p in range(live, len(refs)) if refs[p] > 0]
    holes = [p for p in range(live) if refs[p] <= 0]
    new = refs.copy()
    for x, y in zip(movers, holes):
        to[x] = y
        new[y], new[x] = refs[x], 0
        _copy_page(pool, x, y)
    out = table.copy()
    ok = (table >= 0) & (table < len(refs))
    out[ok] = to[table[ok]]
    return out, new, live, len(movers)


# ---- attention of a window and the first tokens, and of groups that share a prefix ----

def attend_window(pool, layer, batch, q, page, window, sinks, causal=True, scale=None):
    """As attend without lists, of the tokens j < sinks or j > p - window of a token at position p."""
    table = batch[0]
    rows, heads, d = q.shape
    pages, kv = pool["k"].shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    o = np.full((rows, heads, d), np.nan)
    weight, spread = np.zeros((rows, heads, d)), np.zeros((rows, heads))
    for s, (begin, n, start, held) in enumerate(sequences(batch, page, rows)):
        for tok in range(n):
            p, sees = start + tok, visible(start, held, tok, causal)
            j = np.array([x for x in range(sees) if (x < sinks or x > p - window) and
                          0 <= int(table[s, x // page]) < pages], dtype=np.int64)
            for h in range(kv):
                keys, values = (_gather(pool, layer, table[s], j, h, w, page, d) for w in (0, 1))
                for g in range(heads // kv):
                    r, head = begin + tok, h * (heads // kv) + g
                    if not len(j):
                        o[r, head] = 0.0
                        continue
                    w = scale * (keys @ q[r, head])
                    e = np.exp(w - w.max())
                    e /= e.sum()
                    o[r, head] = e @ values
                    weight[r, head] = e @ np.abs(values)
                    spread[r, head] = abs(scale) * (np.abs(keys) @ np.abs(q[r, head])).max()
    return o, weight, spread


def _gather(pool, layer, row, j, h, which, page, d):
    out = np.zeros((len(j), d))
    for lp in np.unique(j // page):
        at = j // page == lp
        out[at] = rows_of(pool, layer, int(row[lp]), h, which, page, d)[j[at] % page]
    return out


def shared_table(batch, first, pages):
    """The table with the shared pages of every group's first sequence in the rows of its others."""
    table = batch[0].copy()
    for g in range(len(pages)):
        for s in range(first[g], first[g + 1]):
            table[s, :pages[g]] = table[first[g], :pages[g]]
    return (table,) + tuple(batch[1:])
