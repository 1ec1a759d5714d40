"""The example of endless conversations, run in small: its attention against the
fp64 reference over the pools that the whole loop left behind, and its pages.

Same bar as the operators' own tests: every output within one bf16 spacing.
"""
import sys
from pathlib import Path

import numpy as np
import pytest

import oracle
from _gpu import check
from oracle import cache as C

pytestmark = pytest.mark.gpu
sys.path.insert(0, str(Path(__file__).resolve().parents[1] / "examples"))


def bits(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def tokens(layer):
    """The layer's K and V pools as float64 [N, P, Hkv, D]."""
    pools = layer.pools
    if layer.kv4:
        k_codes, k_scales, v_codes, v_scales = (p.cpu().numpy() for p in pools)
        return C.kv4_tokens(k_codes, k_scales), C.kv4_tokens(v_codes, v_scales)
    return oracle.bf16_to_f64(bits(pools[0])), oracle.bf16_to_f64(bits(pools[1]))


@pytest.mark.parametrize("cache", ["kv4", "bf16"])
@pytest.mark.parametrize("prompt,steps,window,sinks", [(75, 90, 48, 5), (1, 40, 0, 0), (40, 1, 16, 0)])
def test_loop(gpu_lib, cache, prompt, steps, window, sinks):
    import torch
    import endless_chat
    conv = 2
    r = endless_chat.run(cache, conversations=conv, prompt=prompt, forks=2, steps=steps, window=window, sinks=sinks,
                         layers=2, seed=7, log=lambda s: None)
    pages, page = r["pages"], r["pages"].page
    assert int(pages.lacking) == 0 and torch.isfinite(r["x"].float()).all()
    lens, table = pages.lens.cpu().numpy(), pages.table.cpu().numpy()
    assert (lens == prompt + steps).all()
    # Compaction: the same output, live pages first, each with the holders that the table gives it.
    assert torch.equal(r["before"], r["after"])
    assert torch.equal(r["out"], r["after"])
    count = np.bincount(table[table >= 0], minlength=pages.refcount.shape[0])
    np.testing.assert_array_equal(count, pages.refcount.cpu().numpy())
    assert (count[:r["live"]] > 0).all() and not count[r["live"]:].any()
    # A row holds the pages of its window and its sinks, and no others.
    n = prompt + steps
    seen = C.visible_keys(n, 1, 0, window, sinks)
    for row in table:
        assert set(np.flatnonzero(row >= 0)) == set(np.unique(seen // page))
    k, v = tokens(r["layer"])
    ref = C.attend(bits(r["q"]), k, v, table, lens, 128 ** -0.5, window, sinks)
    check(r["after"].float().cpu().numpy().astype(np.float64), ref, f"{cache} {prompt} {steps} {window} {sinks}")
