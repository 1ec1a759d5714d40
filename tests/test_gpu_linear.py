"""GPU parity of pda_linear against the fp64 oracle, at bounds derived from its roundings."""
import numpy as np
import pytest
import torch

from _ffn import check, f64, gpu, linear_error, values
from oracle import ffn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


def build(b, k, n, gated, bias, residual, seed):
    g = torch.Generator().manual_seed(seed)
    rows = 2 * n if gated else n
    x = values(g, b, k)
    w = values(g, rows, k, std=k ** -0.5)
    return x, w, values(g, rows, std=0.5) if bias else None, values(g, b, n) if residual else None


def run(lib, b, k, n, act="none", gated=False, bias=False, residual=False, f32=False, in_place=False, seed=0):
    x, w, bi, re = build(b, k, n, gated, bias, residual, seed + 131 * b + k + n)
    res = gpu(re)
    out = res if in_place else torch.full((b, n), float("nan"), dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    got = lib.linear(gpu(x), lib.pack_weights(gpu(w)), out, bias=gpu(bi), residual=res, activation=act, gated=gated)
    assert got is out
    torch.cuda.synchronize()
    none = lambda t: None if t is None else f64(t)
    ref = ffn.linear(f64(x), f64(w), none(bi), none(re), act, gated)
    bound = linear_error(f64(x), f64(w), none(bi), none(re), act, gated, ref, f32)
    check(out, ref, bound, f"linear B={b} K={k} N={n} {act} gated={gated}")
    return out


# every form's batch, features off each tile height, k of one tile and of an odd number of them
SHAPES = [(1, 32, 16), (1, 4096, 128), (2, 96, 48), (3, 64, 80), (7, 1024, 1040), (16, 2048, 512), (16, 4096, 8192),
          (17, 992, 336), (31, 512, 2064), (32, 4096, 1024), (33, 640, 272), (48, 2048, 2048), (64, 2048, 128),
          (64, 4096, 4096), (65, 1024, 528), (96, 512, 1040), (101, 2560, 2064), (128, 1024, 16), (129, 96, 4112),
          (200, 4096, 1024), (255, 544, 784), (256, 2048, 4096), (256, 32, 16)]
ids = ["%dx%dx%d" % s for s in SHAPES]


@pytest.mark.parametrize("b,k,n", SHAPES, ids=ids)
def test_plain_product(lib, b, k, n):
    run(lib, b, k, n)


@pytest.mark.parametrize("b,k,n", SHAPES, ids=ids)
def test_gated_with_everything(lib, b, k, n):
    run(lib, b, k, n, act="silu", gated=True, bias=True, residual=True)


@pytest.mark.parametrize("b,k,n", SHAPES, ids=ids)
def test_fp32_out_with_bias(lib, b, k, n):
    run(lib, b, k, n, bias=True, f32=True)


# many output features and more than 64 sequences, little k: each number of column tiles, k of less than a step and off
# a step
STREAM = [(65, 32, 16384), (80, 96, 16400), (81, 1056, 16384), (96, 160, 20480), (112, 640, 16640), (113, 2080, 16384),
          (128, 352, 17408), (129, 1024, 16384), (160, 64, 16400), (161, 544, 20480), (208, 1120, 16384), (209, 96, 18432),
          (256, 992, 16416)]


@pytest.mark.parametrize("b,k,n", STREAM, ids=["%dx%dx%d" % s for s in STREAM])
def test_many_features(lib, b, k, n):
    run(lib, b, k, n, act="gelu_tanh", bias=True)
    run(lib, b, k, n, f32=True, residual=True)


@pytest.mark.parametrize("b,k,n", STREAM, ids=["%dx%dx%d" % s for s in STREAM])
def test_many_features_gated(lib, b, k, n):
    run(lib, b, k, (n // 2 + 15) // 16 * 16, act="silu", gated=True, bias=True, residual=True)


# the form whose activations lie in LDS for all of a workgroup's rows, at each number of column tiles it has a kernel
# for and its next lower one, whole and in 2 to 6 parts of k, k off a step and of less than one, rows off a workgroup's
SHARED = [(33, 96, 61456, 1), (36, 1120, 20480, 1), (64, 544, 28688, 1), (65, 1120, 28672, 1), (80, 6176, 12304, 5),
          (96, 8224, 10256, 3), (96, 32, 20496, 1), (96, 2080, 20496, 1), (113, 544, 61440, 1), (128, 2080, 28688, 1), (129, 2080, 28672, 2),
          (129, 4128, 16400, 3), (129, 6176, 12304, 5), (160, 8224, 10240, 6), (161, 2080, 40960, 1), (208, 8224, 10256, 6),
          (209, 544, 65552, 1), (256, 1056, 40976, 1), (70, 96, 262144, 1)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("b,k,n,parts", SHARED, ids=["%dx%dx%d" % s[:3] for s in SHARED])
def test_shared_activations(lib, b, k, n, parts, gated):
    n = n // 32 * 16 if gated else n
    plan = lib.linear_plan(lib.linear_dims(b, k, n, "silu" if gated else "none", gated))
    assert (plan.row_tiles, plan.col_tiles, plan.col_groups) == (8 if b <= 128 else 16, (b + 15) // 16, 1)
    assert gated or plan.k_splits == parts
    run(lib, b, k, n, act="silu" if gated else "none", gated=gated, bias=True, residual=not gated)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("b,k,n", [(5, 256, 64), (130, 1024, 528)])
def test_activations(lib, act, gated, b, k, n):
    run(lib, b, k, n, act=act, gated=gated, bias=True, residual=not gated)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("b,k,n", [(1, 64, 16), (40, 4096, 1040), (64, 8192, 128), (180, 512, 2064)])
def test_in_place_residual_gives_the_same_bits(lib, gated, b, k, n):
    a = run(lib, b, k, n, act="gelu", gated=gated, residual=True)
    c = run(lib, b, k, n, act="gelu", gated=gated, residual=True, in_place=True)
    assert torch.equal(a, c)


def test_more_features_than_32_bit_offsets_reach(lib):
    # 262144 features x 65536 of k would be 32 GiB; 262144 x 8224 reaches past 4 GiB of weights
    k, n = 8224, 262144
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.empty((n, k), dtype=torch.bfloat16, device="cuda").normal_(0, k ** -0.5, generator=g)
    x = torch.empty((3, k), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    wp = lib.pack_weights(w)
    out = torch.full((3, n), float("nan"), dtype=torch.float32, device="cuda")
    lib.linear(x, wp, out)
    torch.cuda.synchronize()
    for rows in (slice(0, 64), slice(n // 2 - 32, n // 2 + 32), slice(n - 64, n)):
        part = f64(w[rows])
        ref = ffn.linear(f64(x), part)
        check(f64(out[:, rows]), ref, linear_error(f64(x), part, None, None, "none", False, ref, True), f"rows {rows.start}")
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu", "none"])
def test_extreme_products(lib, act):
    # one feature per row of W: products that overflow the exponential, reach infinity, or are NaN
    k, n = 32, 16
    xs = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3.0, -3.0, 9.0, -9.0, 80.0, -80.0, 1e4, -1e4, 1e30, -1e30,
                       float("inf"), float("-inf"), float("nan")]).to(torch.bfloat16)
    x = torch.zeros(len(xs), k, dtype=torch.bfloat16)
    x[:, 5] = xs
    w = torch.zeros(n, k, dtype=torch.bfloat16)
    w[:, 5] = 1.0
    out = torch.empty((len(xs), n), dtype=torch.bfloat16, device="cuda")
    lib.linear(gpu(x), lib.pack_weights(gpu(w)), out, activation=act)
    got = f64(out)[:, 3]
    ref = ffn.activate(f64(xs), act)
    # |z| 2^-24 of the exponential's argument, up to 88 (beyond, the value is 0 or x), and a bf16 half step
    fin = np.isfinite(ref)
    assert np.array_equal(np.isnan(ref), np.isnan(got)) and np.array_equal(ref[~fin & ~np.isnan(ref)], got[~fin & ~np.isnan(ref)])
    assert (np.abs(got - ref)[fin] <= (2.0 ** -8 + 2.0 ** -17) * np.abs(ref[fin]) + 2.0 ** -126).all(), (got, ref)


@pytest.mark.parametrize("n", [64, 16384])
def test_what_is_not_finite_stays_in_its_row(lib, n):
    b, k = 70, 256
    x, w, _, _ = build(b, k, n, False, False, False, 5)
    wp = lib.pack_weights(gpu(w))
    clean = lib.linear(gpu(x), wp, torch.empty((b, n), dtype=torch.bfloat16, device="cuda"))
    x[17, 3], x[69, 255], x[0, 0] = float("nan"), float("inf"), float("-inf")
    got = lib.linear(gpu(x), wp, torch.empty((b, n), dtype=torch.bfloat16, device="cuda"))
    rows = [i for i in range(b) if i not in (0, 17, 69)]
    assert torch.equal(got[rows], clean[rows]) and not torch.isfinite(got[[0, 17, 69]]).any()


@pytest.mark.parametrize("b,k,n,gated,f32", [(100, 512, 10240, True, False), (140, 640, 20480, False, True), (4, 4096, 128, False, True), (64, 4096, 256, True, False), (12, 512, 4096, False, False)])
def test_graph_replay(lib, b, k, n, gated, f32):
    x, w, bi, re = (gpu(t) for t in build(b, k, n, gated, True, True, 7))
    wp = lib.pack_weights(w)
    out = torch.empty((b, n), dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    call = lambda: lib.linear(x, wp, out, bias=bi, residual=re, activation="silu", gated=gated)
    want = call().clone()
    s = torch.cuda.Stream()
    lib.linear_workspace_reserve(lib.linear_dims(b, k, n, "silu", gated, f32), stream=s)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        call()
    for _ in range(3):
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(call(), want)  # eager, on another stream, between the replays


def test_offset_rows_give_the_same_bits(lib):
    # bias, residual and out need only be 2-byte aligned
    b, k, n = 9, 512, 80
    x, w, bi, re = (gpu(t) for t in build(b, k, n, True, True, True, 8))
    wp = lib.pack_weights(w)
    want = lib.linear(x, wp, torch.empty_like(re), bias=bi, residual=re, activation="silu", gated=True)
    buf = torch.empty(3 * (b * n + 2 * n) + 8, dtype=torch.bfloat16, device="cuda")
    bi2 = buf[1:1 + 2 * n].copy_(bi)
    re2 = buf[2 * n + 2:2 * n + 2 + b * n].copy_(re.flatten()).view(b, n)
    out = buf[2 * n + b * n + 3:2 * n + 2 * b * n + 3].view(b, n)
    assert torch.equal(lib.linear(x, wp, out, bias=bi2, residual=re2, activation="silu", gated=True), want)


def test_nothing_else_is_written(lib):
    for b, k, n in ((19, 96, 48), (67, 64, 8208), (200, 128, 8192)):
        x, w, _, _ = (gpu(t) for t in build(b, k, n, True, False, False, 9))
        buf = torch.full((b * n + 512,), 7.0, dtype=torch.bfloat16, device="cuda")
        lib.linear(x, lib.pack_weights(w), buf[256:256 + b * n].view(b, n), gated=True)
        torch.cuda.synchronize()
        assert (buf[:256] == 7).all() and (buf[256 + b * n:] == 7).all()


# each form in use: 1 row and column tile a workgroup, 2 x 1, 2 x 2, the planner's with k split, activations shared
# whole and in 3 to 6 parts
FORMS = [(36, 1024, 256), (40, 2048, 2048), (40, 2048, 4096), (24, 8192, 2560), (70, 1120, 28672), (40, 544, 28672),
         (96, 8224, 10256), (129, 4128, 16400), (129, 8224, 10240)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("b,k,n", FORMS, ids=["%dx%dx%d" % s for s in FORMS])
def test_forms_in_use(lib, b, k, n, gated):
    n = n // 32 * 16 if gated else n
    x, w, bi, re = (gpu(t) for t in build(b, k, n, gated, True, True, 11))
    wp = lib.pack_weights(w)
    kw = dict(bias=bi, activation="silu", gated=gated)
    want = lib.linear(x, wp, torch.empty_like(re), residual=re, **kw)
    # in the residual's place, between guards, captured on a stream whose reserve was for more sequences
    buf = torch.full((b * n + 512,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[256:256 + b * n].view(b, n)
    stream = torch.cuda.Stream()
    lib.linear_workspace_reserve(lib.linear_dims(256, k, n, "silu", gated), stream=stream)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        lib.linear(x, wp, out, residual=out, **kw)
    for _ in range(3):
        out.copy_(re)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(lib.linear(x, wp, torch.empty_like(re), residual=re, **kw), want)
    assert (buf[:256] == 7).all() and (buf[256 + b * n:] == 7).all()
    # what is not finite stays in its sequence
    x[b - 1, k - 1], x[3, 0], x[17, k // 2] = float("inf"), float("nan"), float("-inf")
    got = lib.linear(x, wp, torch.empty_like(re), residual=re, **kw)
    rows = [i for i in range(b) if i not in (3, 17, b - 1)]
    assert torch.equal(got[rows], want[rows]) and torch.isnan(got[3]).all()


def test_empty_batch(lib):
    w = lib.pack_weights(torch.zeros((16, 32), dtype=torch.bfloat16, device="cuda"))
    out = lib.linear(torch.empty((0, 32), dtype=torch.bfloat16, device="cuda"), w,
                     torch.empty((0, 16), dtype=torch.bfloat16, device="cuda"))
    assert out.shape == (0, 16)
