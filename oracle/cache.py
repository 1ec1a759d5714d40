"""fp64 reference of the cache operators: sliding windows with sinks, the
4-bit cache, and the pages of a pool.  Written from the definitions in
include/pda.h, in NumPy, apart from the library and from perf/."""
from __future__ import annotations

import numpy as np

from . import bf16_to_f64

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def visible_keys(length, num_queries, j, window=0, sinks=0):
    """Positions that query j of ``num_queries`` sees: t <= p with, under a
    window W > 0, t > p - W or t < sinks."""
    p = int(length) - int(num_queries) + int(j)
    t = np.arange(max(0, p + 1))
    return t if window <= 0 else t[(t > p - window) | (t < sinks)]


def attend(q, k, v, block_table, context_lens, scale, window=0, sinks=0):
    """q: bf16 bits [B, Tq, Hq, D]; k, v: float64 [N, P, Hkv, D].  A query that
    sees no key gets a zero row.  Returns float64 [B, Tq, Hq, D]."""
    bsz, tq, hq, d = q.shape
    page, hkv = k.shape[1], k.shape[2]
    group = hq // hkv
    sigma = float(np.float32(scale))
    out = np.zeros((bsz, tq, hq, d))
    for b in range(bsz):
        for j in range(tq):
            t = visible_keys(context_lens[b], tq, j, window, sinks)
            if t.size == 0:
                continue
            ids = np.asarray(block_table)[b, t // page]
            for h in range(hq):
                s = sigma * (k[ids, t % page, h // group] @ bf16_to_f64(q[b, j, h]))
                e = np.exp(s - s.max())
                out[b, j, h] = (e / e.sum()) @ v[ids, t % page, h // group]
    return out


def kv4_quantise(x):
    """bf16 bits [..., D] -> codes uint8 [..., D / 32, 16], scales uint8 [..., D / 32]."""
    g = np.asarray(x).reshape(*x.shape[:-1], -1, GROUP)
    top = ((g >> 7) & 255).max(axis=-1).astype(np.int64)
    s = np.where(top == 255, 255, np.maximum(top - 2, 0))
    val = np.where((top == 255)[..., None], 0.0, bf16_to_f64(np.where((top == 255)[..., None], 0, g).astype(np.uint16)))
    units = np.ldexp(np.abs(val), (127 - s)[..., None])  # exact
    away = np.abs(units[..., None] - E2M1)
    best = away.min(axis=-1, keepdims=True)
    code = np.where(away == best, np.where(np.arange(8) % 2 == 0, np.arange(8), np.arange(8) + 100), 1000).min(axis=-1) % 100
    sign = np.where((top == 255)[..., None], 0, g >> 15)
    code = (code | (sign << 3)).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), s.astype(np.uint8)


def kv4_values(codes, scales):
    """What codes [..., 16] and scales [...] stand for as bf16, float64 [..., 32]: exact, but that the
    scales 253 and 254, which quantising never gives, reach past bf16's range (an infinity there)."""
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(*codes.shape[:-1], GROUP)
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    size = E2M1[c & 7] * unit[..., None]
    return np.where(c >= 8, -1.0, 1.0) * np.where(size >= 2.0 ** 128, np.inf, size)


def kv4_cache(cache):
    """A bf16 cache [N, P, Hkv, D] (bits) as codes [N, Hkv, D / 32, P, 16] and
    scales [N, Hkv, D / 32, P]."""
    codes, scales = kv4_quantise(cache)
    return np.ascontiguousarray(codes.transpose(0, 2, 3, 1, 4)), np.ascontiguousarray(scales.transpose(0, 2, 3, 1))


def kv4_tokens(codes, scales):
    """float64 [N, P, Hkv, D] of a 4-bit cache."""
    x = kv4_values(codes, scales).transpose(0, 3, 1, 2, 4)
    return x.reshape(*x.shape[:3], -1)


def kv4_append(codes, scales, new, block_table, context_lens):
    """Copies of one pool's codes and scales with new bf16 rows [B, T, Hkv, D]
    at positions L_b - T + j; a token without a page in the pool goes nowhere."""
    codes, scales = codes.copy(), scales.copy()
    page = codes.shape[3]
    c, s = kv4_quantise(new)
    for b in range(new.shape[0]):
        for j in range(new.shape[1]):
            t = int(context_lens[b]) - new.shape[1] + j
            if t >= 0:
                n = int(block_table[b][t // page])
                if not 0 <= n < len(codes):
                    continue
                codes[n, :, :, t % page] = c[b, j]
                scales[n, :, :, t % page] = s[b, j]
    return codes, scales


def kv4_read(codes, scales, tokens, block_table, context_lens):
    """The last ``tokens`` tokens of each sequence, float64 [B, T, Hkv, D];
    zeros before the first, and where there is no page in the pool."""
    x = kv4_tokens(codes, scales)
    out = np.zeros((len(context_lens), tokens, *x.shape[2:]))
    for b, n in enumerate(context_lens):
        for j in range(tokens):
            t = int(n) - tokens + j
            if t >= 0 and 0 <= block_table[b][t // x.shape[1]] < len(x):
                out[b, j] = x[int(block_table[b][t // x.shape[1]]), t % x.shape[1]]
    return out


# ---------------------------------------------------------------------- pages
def pages_update(table, lens, parents, new_lens, refcount, page, window=0, sinks=0, num_queries=1):
    """Row by row from the rules of pda_pages_update: (table, refcount, copy_src, copy_dst, [taken, lacking])."""
    table = np.asarray(table)
    batch, m = table.shape
    count = np.array(refcount, dtype=np.int64)
    n_pages = len(count)

    def length(b):
        return min(max(int(lens[b]), 0), m * page)

    def entry(b, j):
        e = int(table[b, j])
        return e if 0 <= e < n_pages else -1

    for b in range(batch):
        for j in range(-(-length(b) // page)):
            if entry(b, j) >= 0:
                count[entry(b, j)] -= 1
    rows = len(new_lens)
    out = np.full((rows, m), -1, dtype=np.int32)
    src, dst = np.full(rows, -1, np.int32), np.full(rows, -1, np.int32)
    plans = []
    for r in range(rows):
        b = r if parents is None else int(parents[r])
        has = 0 <= b < batch
        total = min(max(int(new_lens[r]), 0), m * page)
        kept = min(length(b), total) if has else 0
        first_seen = max(0, total - num_queries + 1 - window) if window > 0 else 0
        write = None
        for j in range(-(-kept // page)):
            tokens = range(j * page, (j + 1) * page)
            if tokens[-1] < kept and all(sinks <= t < first_seen for t in tokens):
                continue
            if tokens[-1] >= kept and total > kept:
                write = (j, entry(b, j))
                continue
            out[r, j] = entry(b, j)
            if out[r, j] >= 0:
                count[out[r, j]] += 1
        plans.append((kept, total, write))
    held = count.copy()  # by others than the rows that write
    lowest = {}
    for r, (_, _, write) in enumerate(plans):
        if write and write[1] >= 0:
            lowest.setdefault(write[1], r)
    copies = set()
    for r, (_, _, write) in enumerate(plans):
        if write is None:
            continue
        j, p = write
        if p >= 0 and lowest[p] == r and held[p] == 0:
            out[r, j] = p
            count[p] = 1
        else:
            copies.add(r)
    free = [p for p in range(n_pages) if count[p] == 0]
    taken = lacking = 0

    def fresh():
        nonlocal taken, lacking
        if taken < len(free):
            taken += 1
            count[free[taken - 1]] = 1
            return free[taken - 1]
        lacking += 1
        return -1

    for r, (kept, total, write) in enumerate(plans):
        if r in copies:
            j, p = write
            out[r, j] = fresh()
            if p >= 0 and out[r, j] >= 0:
                src[r], dst[r] = p, out[r, j]
        for j in range(-(-kept // page), -(-total // page)):
            out[r, j] = fresh()
    return out, count.astype(np.int32), src, dst, np.array([taken, lacking], np.int32)


def pages_compact(table, lens, refcount, page):
    """(table, refcount, page_map, copy_src, copy_dst, [live, moved]) of pda_pages_compact."""
    table = np.asarray(table)
    n_pages, m = len(refcount), table.shape[1]
    live = [p for p in range(n_pages) if refcount[p] > 0]
    n = len(live)
    holes = [p for p in range(n) if refcount[p] <= 0]
    movers = [p for p in live if p >= n]
    page_map = np.full(n_pages, -1, np.int32)
    page_map[live] = live
    page_map[movers] = holes
    count = np.zeros(n_pages, np.int32)
    for p in live:
        count[page_map[p]] = refcount[p]
    out = np.full(table.shape, -1, np.int32)
    for b in range(table.shape[0]):
        for j in range(-(-min(max(int(lens[b]), 0), m * page) // page)):
            if 0 <= table[b, j] < n_pages:
                out[b, j] = page_map[table[b, j]]
    src, dst = np.full(n_pages, -1, np.int32), np.full(n_pages, -1, np.int32)
    src[:len(movers)], dst[:len(movers)] = movers, holes
    return out, count, page_map, src, dst, np.array([n, len(movers)], np.int32)
