"""The pages of a pool on the GPU, against the rules written out row by row (integers: equal)."""
import numpy as np
import pytest

from _cache import torch_any
from _gpu import log
from oracle import cache as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


def state(rng, batch, page, maxp, longest, spare, shared=0.2, released=0.1):
    """A table of sequences in shuffled pages, some of which they share or others hold too, some released."""
    lens = rng.integers(0, longest + 1, batch).astype(np.int32)
    pages = -(-lens.astype(int) // page)
    pool = int(pages.sum()) + spare
    ids = rng.permutation(pool)
    table = rng.integers(-3, pool + 3, (batch, maxp)).astype(np.int32)  # whatever lies past a sequence's pages
    count = np.zeros(pool, np.int32)
    at = 0
    for b in range(batch):
        for j in range(pages[b]):
            table[b, j] = ids[at]
            at += 1
            if b and j < pages[b - 1] and rng.random() < shared:
                table[b, j] = table[b - 1, j]
            if rng.random() < released:
                table[b, j] = -1
            if table[b, j] >= 0:
                count[table[b, j]] += 1
    count += (rng.random(pool) < 0.1).astype(np.int32)  # held by others than the table
    return table, lens, count


def update(lib, table, lens, parents, new, count, page, stream=None, **kw):
    import torch
    rows, m = len(new), table.shape[1]
    out = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((rows, m), (len(count),), (rows,), (rows,), (2,))]
    lib.pages_update(torch_any(table), torch_any(lens), None if parents is None else torch_any(parents), torch_any(new),
                     torch_any(count), *out, page_size=page, stream=stream, **kw)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in out]


def same(got, want):
    for name, a, b in zip(("table", "refcount", "src", "dst", "info"), got, want):
        assert np.array_equal(a, b), name


# (batch, rows, page, table width, longest, free pages, window, sinks, query tokens)
UPDATES = [
    (1, 1, 16, 4, 40, 5, 0, 0, 1),
    (5, 9, 16, 12, 150, 60, 0, 0, 1),
    (5, 9, 16, 12, 150, 3, 0, 0, 1),              # too few free pages
    (7, 7, 1, 40, 39, 20, 0, 0, 1),               # one-token pages: nothing is ever half written
    (8, 20, 64, 30, 1900, 200, 500, 70, 2),       # released by the window, sinks kept
    (6, 6, 16, 70, 1100, 40, 33, 0, 1),
    (6, 12, 4, 300, 1190, 900, 100, 9, 4),
    (3, 0, 16, 8, 100, 4, 0, 0, 1),               # nothing goes on
    (0, 4, 16, 8, 0, 40, 0, 0, 1),                # new sequences alone
    (300, 1500, 16, 40, 600, 4000, 0, 0, 1),      # more rows than the scan's workgroup has threads
    (40, 64, 16, 513, 8200, 9000, 4096, 4, 1),
]


@pytest.mark.parametrize("case", UPDATES, ids=[f"B{c[0]}-R{c[1]}-P{c[2]}-F{c[5]}-W{c[6]}-S{c[7]}" for c in UPDATES])
@pytest.mark.parametrize("seed", [0, 1])
def test_update_follows_the_rules(lib, case, seed):
    batch, rows, page, m, longest, spare, window, sinks, nq = case
    rng = np.random.default_rng(seed + 10 * batch)
    table, lens, count = state(rng, batch, page, m, longest, spare)
    parents = rng.integers(-1, batch + 1, rows).astype(np.int32)
    base = np.where((parents >= 0) & (parents < batch), lens[np.clip(parents, 0, max(batch - 1, 0))] if batch else 0, 0)
    new = (base + rng.choice([-40, -1, 0, 1, 1, 1, 5, 17, 100], rows)).astype(np.int32)  # (negative: clamped)
    kw = dict(window=window, sinks=sinks, num_queries=nq)
    log(f"update {case} seed {seed}")
    same(update(lib, table, lens, parents, new, count, page, **kw), C.pages_update(table, lens, parents, new, count, page, **kw))


def test_update_without_parents_continues_each_sequence(lib):
    rng = np.random.default_rng(5)
    table, lens, count = state(rng, 9, 16, 20, 250, 40, shared=0.0)
    new = lens + 1
    same(update(lib, table, lens, None, new, count, 16), C.pages_update(table, lens, None, new, count, 16))
    same(update(lib, table, lens, None, new[:5], count, 16), C.pages_update(table, lens, None, new[:5], count, 16))
    longer = np.concatenate([new, [3, 40]]).astype(np.int32)  # two new sequences
    same(update(lib, table, lens, None, longer, count, 16), C.pages_update(table, lens, None, longer, count, 16))


def test_a_fork_shares_and_copies_the_written_page_once_per_further_row(lib):
    page = 16
    table, lens = np.array([[3, 1, 0, -1]], np.int32), np.array([35], np.int32)
    count = np.array([1, 1, 0, 1, 0, 0, 0, 0], np.int32)
    got = update(lib, table, lens, np.zeros(3, np.int32), np.full(3, 36, np.int32), count, page)
    assert got[0].tolist() == [[3, 1, 0, -1], [3, 1, 2, -1], [3, 1, 4, -1]]
    assert got[1].tolist() == [1, 3, 1, 3, 1, 0, 0, 0]
    assert got[2].tolist() == [-1, 0, 0] and got[3].tolist() == [-1, 2, 4] and got[4].tolist() == [2, 0]


# (batch, page, table width, longest, free pages)
COMPACTS = [(1, 16, 4, 40, 3), (5, 16, 12, 150, 100), (0, 16, 4, 0, 30), (20, 64, 30, 1900, 5000), (64, 16, 513, 8190, 9000),
            (200, 1, 100, 99, 4096), (3, 16, 9, 140, 0)]


@pytest.mark.parametrize("case", COMPACTS, ids=[f"B{c[0]}-P{c[1]}-F{c[4]}" for c in COMPACTS])
def test_compact_follows_the_rules(lib, case):
    import torch
    batch, page, m, longest, spare = case
    rng = np.random.default_rng(batch)
    table, lens, count = state(rng, batch, page, m, longest, spare)
    n = len(count)
    out = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in (table.shape, (n,), (n,), (n,), (n,), (2,))]
    log(f"compact {case}")
    lib.pages_compact(torch_any(table), torch_any(lens), torch_any(count), *out, page_size=page)
    for name, a, b in zip(("table", "refcount", "map", "src", "dst", "info"), out, C.pages_compact(table, lens, count, page)):
        assert np.array_equal(a.cpu().numpy(), b), name


@pytest.mark.parametrize("n", [1, 4095, 4096, 4097, 12289])
@pytest.mark.parametrize("share", [0.0, 0.03, 0.5, 1.0])
def test_compact_at_block_borders(lib, n, share):
    import torch
    rng = np.random.default_rng(n)
    count = (rng.random(n) < share).astype(np.int32) * rng.integers(1, 4, n).astype(np.int32)
    table, lens = np.zeros((0, 3), np.int32), np.zeros(0, np.int32)
    out = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((0, 3), (n,), (n,), (n,), (n,), (2,))]
    lib.pages_compact(torch_any(table), torch_any(lens), torch_any(count), *out, page_size=16)
    for a, b in zip(out, C.pages_compact(table, lens, count, 16)):
        assert np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("shape,dtype", [((50, 16, 8, 128), "bfloat16"), ((50, 2, 2, 16), "uint8"), ((50, 5, 16), "int8"),
                                         ((50, 1024, 8, 64), "uint8"), ((50, 4100, 4), "float32")])
def test_copy(lib, shape, dtype):
    import torch
    rng = np.random.default_rng(2)
    kind = getattr(torch, dtype)
    pools = [torch.randint(0, 255, (*shape[:-1], shape[-1] * torch.empty(0, dtype=kind).element_size()), dtype=torch.uint8,
                           device="cuda").view(kind) for _ in range(3)]
    ids = rng.permutation(shape[0])
    src, dst = ids[:20].astype(np.int32), ids[20:40].astype(np.int32)
    src[3], dst[7], src[11], dst[12] = -1, -1, shape[0], shape[0] + 5
    want = [p.view(torch.uint8).clone() for p in pools]
    for limit in (None, 5, 0, -2, 100):
        count = None if limit is None else torch.tensor([limit], dtype=torch.int32, device="cuda")
        got = [p.clone() for p in pools]
        lib.pages_copy(got, torch_any(src), torch_any(dst), count=count)
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            expect = w.clone()
            for a, b in list(zip(src, dst))[:20 if limit is None else max(0, min(20, limit))]:
                if 0 <= a < shape[0] and 0 <= b < shape[0]:
                    expect[int(b)] = w[int(a)]
            assert torch.equal(g.view(torch.uint8), expect), limit


def test_copy_of_more_pools_than_a_launch_takes(lib):
    import torch
    pools = [torch.full((6, 2, 16), i % 250, dtype=torch.uint8, device="cuda") for i in range(300)]
    for p in pools:
        p[4] = 251
    lib.pages_copy(pools, torch_any(np.array([4], np.int32)), torch_any(np.array([1], np.int32)))
    for i, p in enumerate(pools):
        assert (p[1] == 251).all() and (p[0] == i % 250).all()


def test_copy_past_four_gigabytes(lib):
    import torch
    pool = torch.zeros((150_000, 32768), dtype=torch.uint8, device="cuda")
    pool[149_999] = 9
    pool[70_001] = 8
    lib.pages_copy([pool], torch_any(np.array([149_999, 70_001], np.int32)), torch_any(np.array([3, 149_998], np.int32)))
    assert (pool[3] == 9).all() and (pool[149_998] == 8).all() and (pool[4] == 0).all()


def test_graph_replays_on_another_stream(lib):
    import torch
    rng = np.random.default_rng(8)
    table, lens, count = state(rng, 9, 16, 30, 400, 90)
    rows, m, n = 18, 30, len(count)
    parents, new = np.arange(18, dtype=np.int32) % 9, lens[np.arange(18) % 9] + 1
    want = C.pages_update(table, lens, parents, new, count, 16)
    dev = [torch_any(x) for x in (table, lens, parents, new.astype(np.int32), count)]
    out = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((rows, m), (n,), (rows,), (rows,), (2,))]
    pool = torch.randint(0, 255, (n, 48), dtype=torch.uint8, device="cuda")
    first = pool.clone()
    s = torch.cuda.Stream()
    lib.pages_workspace_reserve(rows, n, stream=s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        lib.pages_update(*dev, *out, page_size=16)
        lib.pages_copy([pool], out[2], out[3])
    for rep in range(4):
        for t in out:
            t.fill_(5)
        pool.copy_(first)
        update(lib, table[:3], lens[:3], None, lens[:3], count, 16)
        g.replay()
        torch.cuda.synchronize()
        same([t.cpu().numpy() for t in out], want)
        expect = first.clone()
        for a, b in zip(want[2], want[3]):
            if b >= 0:
                expect[int(b)] = first[int(a)]
        assert torch.equal(pool, expect), rep


def test_refusals(lib):
    import torch
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    table, lens, new, count = i(2, 4), i(2), i(3), i(8)
    outs = [i(3, 4), i(8), i(3), i(3), i(2)]
    with pytest.raises(ValueError, match="copy_dst"):
        lib.pages_update(table, lens, None, new, count, *outs[:3], i(2), outs[4], page_size=16)
    with pytest.raises(ValueError, match="table_out"):
        lib.pages_update(table, lens, None, new, count, i(3, 5), *outs[1:], page_size=16)
    with pytest.raises(lib.PdaError, match="refcount_out overlaps refcount"):
        lib.pages_update(table, lens, None, new, count, outs[0], count, *outs[2:], page_size=16)
    with pytest.raises(lib.PdaError, match="page_size"):
        lib.pages_update(table, lens, None, new, count, *outs, page_size=12)
    with pytest.raises(TypeError, match="refcount"):
        lib.pages_compact(table, lens, count.long(), i(2, 4), i(8), i(8), i(8), i(8), i(2), page_size=16)
    with pytest.raises(ValueError, match="pool 1"):
        lib.pages_copy([torch.zeros((4, 16), device="cuda"), torch.zeros((5, 16), device="cuda")], i(1), i(1))
    with pytest.raises(ValueError, match="contiguous"):
        lib.pages_copy([torch.zeros((4, 32), device="cuda")[:, ::2]], i(1), i(1))
    with pytest.raises(lib.PdaError, match="multiple of 16"):
        lib.pages_copy([torch.zeros((4, 3), device="cuda")], i(1), i(1))
