"""Helpers for the GPU tests of the cache operators."""
import numpy as np

import workloads as W

NAN = np.uint16(0x7FC1)


def torch_bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16).cuda()


def torch_any(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def hide(w, num_queries, window, sinks):
    """NaN in every cached token of workload w that no query sees, and its pages without any other
    released (-1 in the table)."""
    page = w.k_cache.shape[1]
    if window <= 0:
        return w
    for b, n in enumerate(w.context_lens):
        n = int(n)
        first = max(0, n - num_queries + 1 - window)
        pinned = min(sinks, first)
        for t in range(pinned, first):
            w.k_cache[w.block_table[b, t // page], t % page] = NAN
            w.v_cache[w.block_table[b, t // page], t % page] = NAN
        for j in range(-(-n // page)):
            if j * page >= pinned and (j + 1) * page <= first:
                w.block_table[b, j] = -1
    return w


def build(lens, hq, hkv, d, page, seed, num_queries=1, window=0, sinks=0, **kw):
    w = W.build(lens, hq, hkv, d, page, seed=seed, pool="holes:0.2", num_queries=num_queries, **kw)
    if w.q.ndim == 3:
        w.q = w.q[:, None]
    w.k_cache, w.v_cache, w.block_table = w.k_cache.copy(), w.v_cache.copy(), w.block_table.copy()
    return hide(w, num_queries, window, sinks)
