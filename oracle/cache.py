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
    at positions L_b - T + j."""
    codes, scales = codes.copy(), scales.copy()
    page = codes.shape[3]
    c, s = kv4_quantise(new)
    for b in range(new.shape[0]):
        for j in range(new.shape[1]):
            t = int(context_lens[b]) - new.shape[1] + j
            if t >= 0:
                n = int(block_table[b][t // page])
                codes[n, :, :, t % page] = c[b, j]
                scales[n, :, :, t % page] = s[b, j]
    return codes, scales


def kv4_read(codes, scales, tokens, block_table, context_lens):
    """The last ``tokens`` tokens of each sequence, float64 [B, T, Hkv, D]; zeros before the first."""
    x = kv4_tokens(codes, scales)
    out = np.zeros((len(context_lens), tokens, *x.shape[2:]))
    for b, n in enumerate(context_lens):
        for j in range(tokens):
            t = int(n) - tokens + j
            if t >= 0:
                out[b, j] = x[int(block_table[b][t // x.shape[1]]), t % x.shape[1]]
    return out
