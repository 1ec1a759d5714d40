"""The cache operators at the borders of their forms: page updates on both sides of the one-launch
placement's limits, and values that are not finite and that only some queries of a sequence see."""
import numpy as np
import pytest

import oracle
from _cache import build, torch_any, torch_bf16
from _gpu import check, log
from oracle import cache as C
from test_gpu_kv4 import quantised
from test_gpu_kv4 import run as run_kv4
from test_gpu_pages import same, state, update
from test_gpu_sink import run as run_sink

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


# (rows, table width, pages of the pool): 60 KB of places and starts, 256 workgroups of 1024 entries,
# 1024 rows
BORDERS = [(32, 40, 15328), (32, 40, 15329), (1024, 16, 14336), (1024, 16, 14337), (1024, 256, 9000), (1024, 257, 9000),
           (1025, 16, 9000)]


@pytest.mark.parametrize("rows,m,pages", BORDERS)
def test_update_at_the_borders_of_the_one_launch_placement(lib, rows, m, pages):
    rng = np.random.default_rng(rows + pages)
    table, lens, count = state(rng, 20, 16, m, 240, 0)
    count = np.concatenate([count, np.zeros(pages - len(count), np.int32)])
    parents = rng.integers(-1, 20, rows).astype(np.int32)
    new = (np.where(parents >= 0, lens[np.maximum(parents, 0)], 0) + rng.integers(0, 18, rows)).astype(np.int32)
    log(f"update rows={rows} width={m} pages={pages}")
    same(update(lib, table, lens, parents, new, count, 16), C.pages_update(table, lens, parents, new, count, 16))


def test_update_of_nothing(lib):
    none = np.zeros(0, np.int32)
    got = update(lib, np.zeros((0, 4), np.int32), none, None, none, np.array([0, 2, 0, 1], np.int32), 16)
    assert got[1].tolist() == [0, 2, 0, 1] and got[4].tolist() == [0, 0]


# the update in one launch: 60 KB of counts, writers and rows, 8192 entries of both tables
@pytest.mark.parametrize("rows,m,pages", [(32, 40, 7506), (32, 40, 7507), (44, 128, 900), (45, 128, 900), (44, 129, 900),
                                          (44, 100, 900), (480, 16, 3600), (492, 16, 3600), (493, 16, 3600), (1, 16, 300)])
def test_update_at_the_borders_of_one_launch(lib, rows, m, pages):
    test_update_at_the_borders_of_the_one_launch_placement(lib, rows, m, pages)


# compaction in one launch: 8192 pages, 262144 pages and entries
@pytest.mark.parametrize("pages,batch,m", [(8191, 20, 16), (8192, 20, 16), (8193, 20, 16), (70000, 20, 16), (4096, 16, 16128),
                                           (4096, 16, 16129), (63, 3, 16), (64, 3, 16), (65, 3, 16)])
@pytest.mark.parametrize("live", [0.1, 0.9, 1.0])
def test_compact_at_the_borders_of_one_launch(lib, pages, batch, m, live):
    import torch
    rng = np.random.default_rng(pages + m)
    count = (rng.random(pages) < live).astype(np.int32) * rng.integers(1, 4, pages).astype(np.int32)
    lens = rng.integers(0, 16 * min(m, 40), batch).astype(np.int32)
    table = rng.integers(-2, pages + 2, (batch, m)).astype(np.int32)
    out = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in (table.shape, (pages,), (pages,), (pages,), (pages,), (2,))]
    log(f"compact pages={pages} batch={batch} width={m} live={live}")
    lib.pages_compact(torch_any(table), torch_any(lens), torch_any(count), *out, page_size=16)
    for name, a, b in zip(("table", "refcount", "map", "src", "dst", "info"), out, C.pages_compact(table, lens, count, 16)):
        assert np.array_equal(a.cpu().numpy(), b), name


# (head_dim, Hq, Hkv, page, lengths, query tokens, window, sinks): the last tokens of a sequence, the far
# end of a window and the sinks lie in different steps, in one step, in a sequence shorter than its queries
SHAPES = [
    (128, 32, 8, 16, [500, 66, 2, 3001], 4, 100, 5),
    (128, 8, 1, 32, [64, 33, 4000], 2, 20, 3),
    (64, 16, 4, 16, [200, 40, 5], 3, 37, 2),
    (256, 12, 4, 16, [300, 31, 1], 5, 64, 4),
    (128, 32, 8, 16, [300, 7], 4, 0, 0),
    (64, 4, 2, 64, [129, 3], 8, 0, 0),
]


def partly_seen(n, tq, window, sinks):
    """The tokens that some, but not all, of a sequence's queries see."""
    seen = [set(C.visible_keys(n, tq, j, window, sinks).tolist()) for j in range(tq)]
    return sorted(set().union(*seen) - set.intersection(*seen))


def compare(got, want, what):
    finite = np.isfinite(want)
    assert not finite.all() and np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), what
    check(np.where(finite, got, 0), np.where(finite, want, 0), what)


IDS = [f"D{c[0]}-{c[1]}:{c[2]}-T{c[5]}-W{c[6]}-S{c[7]}" for c in SHAPES]


@pytest.mark.parametrize("pick", [0, 1, -1, None])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_kv4_values_reach_only_the_queries_that_see_them(lib, shape, pick):
    d, hq, hkv, page, lens, tq, window, sinks = shape
    w = build(lens, hq, hkv, d, page, seed=sum(lens), num_queries=tq, window=window, sinks=sinks)
    kc, ks, vc, vs = (t.copy() for t in quantised(w))
    for b, n in enumerate(lens):
        part = partly_seen(n, tq, window, sinks)
        for i, t in enumerate(part if pick is None else part[pick:][:1]):
            at = int(w.block_table[b, t // page])
            if (b + i) % 2:
                vs[at, :, 0, t % page] = 255                  # NaN
            else:
                vs[at, :, 1, t % page] = 254                  # an infinity among zeros
                vc[at, :, 1, t % page] = 0
                vc[at, :, 1, t % page, 3] = 0x70 if i % 4 else 0x0F
    cache = (kc, ks, vc, vs)
    want = C.attend(w.q, C.kv4_tokens(kc, ks), C.kv4_tokens(vc, vs), w.block_table, w.context_lens, w.scale, window, sinks)
    log(f"kv4 partly seen {shape} {pick}")
    compare(run_kv4(lib, w, cache, window, sinks), want, "kv4")


@pytest.mark.parametrize("pick", [0, 1, -1, None])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[6]] + [(128, 16, 4, 4, [200, 40, 5], 3, 37, 2), (64, 4, 2, 1, [90, 3], 2, 20, 6)])
def test_bf16_values_reach_only_the_queries_that_see_them(lib, shape, pick):
    d, hq, hkv, page, lens, tq, window, sinks = shape
    w = build(lens, hq, hkv, d, page, seed=sum(lens), num_queries=tq, window=window, sinks=sinks)
    for b, n in enumerate(lens):
        part = partly_seen(n, tq, window, sinks)
        for i, t in enumerate(part if pick is None else part[pick:][:1]):
            row = w.v_cache[int(w.block_table[b, t // page]), t % page]
            row[:, (7 * b + 11 * i + np.arange(hkv)) % d] = (0x7FC0, 0x7F80, 0xFF80)[(b + i) % 3]
    want = C.attend(w.q, oracle.bf16_to_f64(w.k_cache), oracle.bf16_to_f64(w.v_cache), w.block_table, w.context_lens, w.scale,
                    window, sinks)
    log(f"bf16 partly seen {shape} {pick}")
    compare(run_sink(lib, w, window, sinks), want, "sink")


def test_keys_that_are_not_finite_reach_only_the_queries_that_see_them(lib):
    lens, tq, window, sinks = [500, 66], 3, 100, 5
    w = build(lens, 32, 8, 128, 16, seed=5, num_queries=tq, window=window, sinks=sinks)
    for b, n in enumerate(lens):
        for t in partly_seen(n, tq, window, sinks)[-1:]:
            w.k_cache[int(w.block_table[b, t // 16]), t % 16, ::2, 9] = 0x7FC0
    cache = quantised(w)
    want = C.attend(w.q, C.kv4_tokens(*cache[:2]), C.kv4_tokens(*cache[2:]), w.block_table, w.context_lens, w.scale, window, sinks)
    compare(run_kv4(lib, w, cache, window, sinks), want, "kv4 keys")
    want = C.attend(w.q, oracle.bf16_to_f64(w.k_cache), oracle.bf16_to_f64(w.v_cache), w.block_table, w.context_lens, w.scale,
                    window, sinks)
    compare(run_sink(lib, w, window, sinks), want, "sink keys")


# (head_dim, Hq, Hkv, page, batch, longest): each side of the rules for whole sequences and for the steps
# of a wave
PLANS = [(128, 32, 8, 16, 1, 512), (128, 32, 8, 16, 1, 528), (128, 8, 2, 16, 70, 1024), (128, 8, 2, 16, 70, 1040),
         (128, 8, 8, 16, 100, 512), (128, 8, 8, 16, 100, 528), (128, 3, 3, 16, 90, 300), (128, 4, 4, 16, 24, 1000),
         (128, 4, 4, 16, 23, 1000), (256, 4, 4, 16, 16, 256), (256, 4, 4, 16, 16, 272), (256, 4, 4, 16, 32, 1000),
         (256, 4, 4, 16, 64, 1024), (256, 4, 4, 16, 140, 130), (64, 2, 2, 16, 200, 500), (64, 2, 2, 16, 1, 8208),
         (128, 4, 2, 16, 1, 12000), (128, 8, 8, 16, 1, 8192), (256, 3, 1, 16, 1, 12000)]


@pytest.mark.parametrize("d,hq,hkv,page,batch,longest", PLANS)
def test_kv4_at_the_borders_of_its_plans(lib, d, hq, hkv, page, batch, longest):
    rng = np.random.default_rng(batch + longest)
    lens = rng.integers(0, 120, batch)
    lens[batch // 2] = longest
    w = build(lens.tolist(), hq, hkv, d, page, seed=batch + longest)
    cache = quantised(w)
    want = C.attend(w.q, C.kv4_tokens(*cache[:2]), C.kv4_tokens(*cache[2:]), w.block_table, w.context_lens, w.scale)
    log(f"kv4 plan D={d} {hq}:{hkv} B={batch} longest={longest}")
    check(run_kv4(lib, w, cache), want, "plan")


@pytest.mark.parametrize("d,hq,hkv,page,batch,longest", PLANS[::2] + [(128, 32, 8, 16, 40, 3000), (128, 8, 8, 16, 3, 40000)])
def test_a_reserve_covers_every_plan_of_its_sizes(lib, d, hq, hkv, page, batch, longest):
    import torch
    rng = np.random.default_rng(longest)
    lens = rng.integers(0, 120, batch)
    lens[0] = longest
    w = build(lens.tolist(), hq, hkv, d, page, seed=longest, poison=False)
    cache = [torch_any(t) for t in quantised(w)]
    table, lens = torch_any(w.block_table), torch_any(w.context_lens)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    lib.release_workspaces()
    lib.kv4_workspace_reserve(batch, hq, hkv, d, page, table.shape[1], stream=s)
    most = 16 // (hq // hkv)
    calls = [(tq, window, sinks) for tq in sorted({1, most}) for window, sinks in ((0, 0), (100, 4), (1000, 300))]
    qs = [torch.randn((batch, tq, hq, d), device="cuda").bfloat16() for tq, _, _ in calls]
    outs = [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        for (_, window, sinks), q, out in zip(calls, qs, outs):
            lib.paged_decode_attention_kv4(q, *cache, table, lens, out, float(w.scale), window=window, sinks=sinks)
    for rep in range(3):
        for out in outs:
            out.zero_()
        g.replay()
        torch.cuda.synchronize()
        for (_, window, sinks), q, out in zip(calls, qs, outs):
            eager = torch.zeros_like(q)
            lib.paged_decode_attention_kv4(q, *cache, table, lens, eager, float(w.scale), window=window, sinks=sinks)
            torch.cuda.synchronize()
            assert torch.equal(out, eager), (rep, window, sinks)


# Batches whose prefix leaves LDS for one workgroup a CU only, of 12, 8 or 4 waves, with a sequence that is
# split.
@pytest.mark.parametrize("d,hq,hkv,batch,longest,tq,window", [(128, 8, 2, 3000, 2000, 1, 0), (128, 4, 1, 8192, 40, 1, 0),
                                                              (128, 4, 4, 2500, 5000, 2, 60), (64, 4, 2, 5000, 3000, 1, 0),
                                                              (256, 2, 1, 4000, 1500, 1, 0), (128, 3, 3, 3500, 700, 1, 0)])
def test_kv4_very_large_batches(lib, d, hq, hkv, batch, longest, tq, window):
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, 20, batch)
    lens[batch // 3] = longest
    w = build(lens.tolist(), hq, hkv, d, 16, seed=batch, num_queries=tq, window=window, sinks=4)
    cache = quantised(w)
    want = C.attend(w.q, C.kv4_tokens(*cache[:2]), C.kv4_tokens(*cache[2:]), w.block_table, w.context_lens, w.scale, window, 4)
    log(f"kv4 batch={batch} D={d} {hq}:{hkv} longest={longest}")
    check(run_kv4(lib, w, cache, window, 4), want, "batch")
