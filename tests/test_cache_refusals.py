"""Argument checks of the cache operators' entry points (before any HIP call, so no GPU)."""
import ctypes

import pytest

from paper_2606_07665_amd import binding as B

NULL, SHAPE, UNSUPPORTED, SCALE, ALIGN = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    return B.load()


def kv4(lib, ptrs=None, batch=2, hq=32, hkv=8, d=128, p=16, n=64, maxp=8, nq=1, window=0, sinks=0, scale=0.1):
    return lib.paged_decode_attention_kv4(*(ptrs or [16] * 8), batch, hq, hkv, d, p, n, maxp, nq, window, sinks,
                                          ctypes.c_float(scale), None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(ptrs=[16] * 2 + [0] + [16] * 5), NULL, "NULL"),
    (dict(ptrs=[8] + [16] * 7), ALIGN, "16-byte"),
    (dict(ptrs=[16, 24] + [16] * 6), ALIGN, "k_codes"),
    (dict(ptrs=[16] * 6 + [18, 16]), ALIGN, "4-byte"),
    (dict(batch=-1), SHAPE, "batch"),
    (dict(batch=8193), UNSUPPORTED, "batch"),
    (dict(hkv=7), SHAPE, "multiple"),
    (dict(d=96), UNSUPPORTED, "head_dim"),
    (dict(p=8), UNSUPPORTED, "page_size"),
    (dict(p=24), UNSUPPORTED, "page_size"),
    (dict(n=0), SHAPE, "num_pages"),
    (dict(nq=0), SHAPE, "num_queries"),
    (dict(nq=5), UNSUPPORTED, "exceeds 16"),
    (dict(window=-1), SHAPE, "window"),
    (dict(window=1, sinks=-1), SHAPE, "num_sinks"),
    (dict(scale=float("nan")), SCALE, "finite"),
])
def test_kv4_attention(lib, kw, code, text):
    assert kv4(lib, **kw) == code
    assert text in B.last_error()


def test_empty_batches_are_no_ops(lib):
    assert kv4(lib, batch=0, ptrs=[0] * 8) == 0
    for fn in (lib.pda_kv4_append, lib.pda_kv4_read):
        assert fn(*[0] * 8, 0, 1, 8, 128, 16, 4, 8, None) == 0


@pytest.mark.parametrize("kw,code,text", [
    (dict(sinks=-1), SHAPE, "num_sinks"),
    (dict(window=-1), SHAPE, "window"),
    (dict(nq=17), UNSUPPORTED, "exceeds 16"),
    (dict(ptr=0), NULL, "NULL"),
    (dict(ptr=8), ALIGN, "aligned"),
])
def test_sink_attention(lib, kw, code, text):
    a = dict(dict(ptr=16, nq=1, window=64, sinks=4), **kw)
    assert lib.paged_decode_attention_sink(*[a["ptr"]] * 6, 2, 8, 8, 128, 16, 64, 8, a["nq"], a["window"], a["sinks"],
                                           ctypes.c_float(0.1), None) == code
    assert text in B.last_error()


@pytest.mark.parametrize("call", ["pda_kv4_append", "pda_kv4_read"])
@pytest.mark.parametrize("kw,code,text", [
    (dict(ptrs=[16] * 5 + [0] + [16] * 2), NULL, "NULL"),
    (dict(ptrs=[18] + [16] * 7), ALIGN, "16-byte"),
    (dict(ptrs=[16] * 7 + [2]), ALIGN, "4-byte"),
    (dict(t=0), SHAPE, "num_tokens"),
    (dict(t=(1 << 20) + 1), SHAPE, "num_tokens"),
    (dict(t=1 << 20, hkv=9), UNSUPPORTED, "2^30"),
    (dict(p=8), UNSUPPORTED, "page_size"),
    (dict(d=32), UNSUPPORTED, "head_dim"),
    (dict(n=-1), SHAPE, "num_pages"),
])
def test_kv4_tokens(lib, call, kw, code, text):
    a = dict(dict(ptrs=[16] * 8, t=1, hkv=8, d=128, p=16, n=4), **kw)
    assert getattr(lib, call)(*a["ptrs"], 2, a["t"], a["hkv"], a["d"], a["p"], a["n"], 8, None) == code
    assert text in B.last_error()


def test_kv4_reserve(lib):
    assert lib.pda_kv4_workspace_reserve(2, 32, 8, 128, 8, 8, None) == UNSUPPORTED
    assert lib.pda_kv4_workspace_reserve(2, 32, 7, 128, 16, 8, None) == SHAPE
    assert lib.pda_kv4_workspace_reserve(0, 32, 8, 128, 16, 8, None) == 0


# ---------------------------------------------------------------------- pages
LAYOUT = 8


def spread(n, size=1 << 20):
    return [(1 + i) * size for i in range(n)]


@pytest.mark.parametrize("kw,code,text", [
    (dict(null=0), NULL, "block_table"),
    (dict(null=3), NULL, "new_lens"),
    (dict(null=9), NULL, "info"),
    (dict(odd=5), ALIGN, "table_out"),
    (dict(batch=-1), SHAPE, "batch"),
    (dict(rows=8193), UNSUPPORTED, "batch"),
    (dict(p=3), UNSUPPORTED, "page_size"),
    (dict(n=0), SHAPE, "num_pages"),
    (dict(n=(1 << 24) + 1), UNSUPPORTED, "num_pages"),
    (dict(nq=0), SHAPE, "num_queries"),
    (dict(window=-1), SHAPE, "window"),
    (dict(sinks=-1), SHAPE, "num_sinks"),
    (dict(same=(5, 0)), LAYOUT, "table_out overlaps block_table"),
    (dict(same=(8, 7)), LAYOUT, "copy_dst overlaps copy_src"),
])
def test_pages_update(lib, kw, code, text):
    a = dict(dict(batch=2, rows=3, p=16, n=64, maxp=8, nq=1, window=0, sinks=0), **kw)
    ptr = spread(10)
    if "null" in a:
        ptr[a["null"]] = 0
    if "odd" in a:
        ptr[a["odd"]] += 2
    if "same" in a:
        ptr[a["same"][0]] = ptr[a["same"][1]]
    assert lib.pda_pages_update(*ptr, a["batch"], a["rows"], a["p"], a["n"], a["maxp"], a["nq"], a["window"], a["sinks"],
                                None) == code
    assert text in B.last_error()


@pytest.mark.parametrize("null,odd,same,code,text", [
    (2, None, None, NULL, "refcount"), (None, 8, None, ALIGN, "info"), (None, None, (4, 2), LAYOUT, "refcount_out"),
    (None, None, (3, 0), LAYOUT, "table_out")])
def test_pages_compact(lib, null, odd, same, code, text):
    ptr = spread(9)
    if null is not None:
        ptr[null] = 0
    if odd is not None:
        ptr[odd] += 1
    if same:
        ptr[same[0]] = ptr[same[1]]
    assert lib.pda_pages_compact(*ptr, 2, 16, 64, 8, None) == code
    assert text in B.last_error()


@pytest.mark.parametrize("kw,code,text", [
    (dict(data=0), NULL, "pool 0"),
    (dict(data=8), ALIGN, "16-byte"),
    (dict(size=24), ALIGN, "multiple of 16"),
    (dict(size=0), SHAPE, "page_bytes"),
    (dict(src=0), NULL, "NULL"),
    (dict(src=2), ALIGN, "copy_src"),
    (dict(most=-1), SHAPE, "max_copies"),
    (dict(most=1 << 24, size=1 << 15), UNSUPPORTED, "max_copies"),
    (dict(n=0), SHAPE, "num_pages"),
    (dict(pools=-1), SHAPE, "num_pools"),
])
def test_pages_copy(lib, kw, code, text):
    a = dict(dict(data=16, size=32, src=16, most=4, n=8, pools=1), **kw)
    pools = (B.Pool * 1)(B.Pool(a["data"], a["size"]))
    assert lib.pda_pages_copy(pools, a["pools"], a["src"], 16, None, a["most"], a["n"], None) == code
    assert text in B.last_error()


def test_pages_no_ops(lib):
    assert lib.pda_pages_copy(None, 0, None, None, None, 5, 8, None) == 0
    assert lib.pda_pages_copy(None, 3, None, None, None, 0, 8, None) == 0
    assert lib.pda_pages_workspace_reserve(-1, 5, None) == SHAPE
    assert lib.pda_pages_workspace_reserve(1, 0, None) == SHAPE
