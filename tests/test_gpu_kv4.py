"""GPU parity of the 4-bit cache (append, read, attention) through the C ABI, against the fp64 reference.

Append and read are exact: whole pools are compared byte for byte, values bit
for bit.  Attention: keys and values are exact in bf16, scores and sums are
fp32 and each probability is carried to ~2^-17, so what is left is the
output's own rounding (half a bf16 spacing) and an fp32 error far below the
other half: one spacing, as for the bf16 cache.
"""
import numpy as np
import pytest

import oracle
import workloads as W
from _cache import build, torch_any, torch_bf16
from _gpu import check, log
from oracle import cache as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


def quantised(w):
    """(k codes, k scales, v codes, v scales) of workload w's caches."""
    return (*C.kv4_cache(w.k_cache), *C.kv4_cache(w.v_cache))


def run(lib, w, cache, window=0, sinks=0, scale=None, stream=None):
    import torch
    q = torch_bf16(w.q)
    out = torch.full(tuple(q.shape), float("nan"), dtype=torch.bfloat16, device="cuda")
    lib.paged_decode_attention_kv4(q, *(torch_any(t) for t in cache), torch_any(w.block_table), torch_any(w.context_lens), out,
                                   float(w.scale if scale is None else scale), window=window, sinks=sinks, stream=stream)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


def ref(w, cache, window=0, sinks=0, scale=None):
    return C.attend(w.q, C.kv4_tokens(*cache[:2]), C.kv4_tokens(*cache[2:]), w.block_table, w.context_lens,
                    w.scale if scale is None else scale, window, sinks)


# ----------------------------------------------------------- append and read
def odd_bits(rng, shape):
    """Rows of every size: normal, tiny, huge, zero, subnormal, infinite and NaN groups."""
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-80, 80, (*shape[:-1], 1)))
    b = W.f32_to_bf16_bits(x.astype(np.float32))
    g = b.reshape(*shape[:-1], -1, 32)
    kind = rng.integers(0, 12, g.shape[:-1])
    g[kind == 0] = 0
    g[kind == 1] &= 0x807F            # subnormals
    g[kind == 2, 7] = 0xFF80          # an infinity
    g[kind == 3, 30] = 0x7FC0         # a NaN
    g[kind == 4] = np.where(g[kind == 4] & 1, 0x40A0, 0x3F40)  # ties in a group of 5.0 and 0.75
    return b


# (head_dim, kv heads, page, tokens, lengths)
APPENDS = [
    (128, 8, 16, 1, [1, 16, 17, 300, 0]),
    (128, 8, 16, 7, [7, 3, 0, 33, 500]),           # fewer cached than new tokens
    (128, 2, 16, 8, [8, 9, 24, 1000]),
    (128, 8, 32, 33, [33, 40, 700]),
    (64, 2, 16, 1, [5, 64]),
    (64, 2, 64, 100, [100, 131, 99]),
    (256, 4, 16, 9, [9, 50, 1]),
    (256, 1, 1024, 300, [1200, 300]),
    (128, 1, 128, 1025, [1025, 2000]),
]


@pytest.mark.parametrize("d,hkv,page,tokens,lens", APPENDS, ids=[f"D{a[0]}-H{a[1]}-P{a[2]}-T{a[3]}" for a in APPENDS])
def test_append_and_read_are_exact(lib, d, hkv, page, tokens, lens):
    import torch
    rng = np.random.default_rng(d + tokens)
    w = build(lens, hkv, hkv, d, page, seed=1 + tokens)
    n = w.k_cache.shape[0]
    codes, scales = rng.integers(0, 256, (2, n, hkv, d // 32, page, 16), np.uint8), rng.integers(0, 256, (2, n, hkv, d // 32, page), np.uint8)
    new = [odd_bits(rng, (len(lens), tokens, hkv, d)) for _ in range(2)]
    log(f"append D={d} H={hkv} P={page} T={tokens}")
    dev = [torch_any(x) for x in (codes[0], scales[0], codes[1], scales[1])]
    table, cl = torch_any(w.block_table), torch_any(w.context_lens)
    lib.kv4_append(torch_bf16(new[0]), torch_bf16(new[1]), *dev, table, cl)
    back = [torch.full((len(lens), tokens, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib.kv4_read(*back, *dev, table, cl)
    torch.cuda.synchronize()
    for i in range(2):
        c, s = C.kv4_append(codes[i], scales[i], new[i], w.block_table, w.context_lens)
        assert np.array_equal(dev[2 * i].cpu().numpy(), c) and np.array_equal(dev[2 * i + 1].cpu().numpy(), s)
        want = C.kv4_read(c, s, tokens, w.block_table, w.context_lens)
        got = back[i].float().cpu().numpy().astype(np.float64)
        assert np.array_equal(got, want, equal_nan=True)


def test_read_of_every_scale_and_code(lib):
    import torch
    codes = np.broadcast_to(np.arange(256, dtype=np.uint8).reshape(16, 16), (16, 1, 2, 16, 16)).copy()  # 16 pages of 16 slots
    scales = np.arange(256, dtype=np.uint8).reshape(16, 1, 1, 16).repeat(2, axis=2)
    lens = torch.tensor([256], dtype=torch.int32, device="cuda")
    table = torch.arange(16, dtype=torch.int32, device="cuda")[None]
    out = [torch.empty((1, 256, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib.kv4_read(*out, torch_any(codes), torch_any(scales), torch_any(codes), torch_any(scales), table, lens)
    want = C.kv4_read(codes, scales, 256, np.arange(16)[None], [256])
    for o in out:
        assert np.array_equal(o.float().cpu().numpy().astype(np.float64), want, equal_nan=True)


# ----------------------------------------------------------------- attention
# (head_dim, Hq, Hkv, page, lengths, query tokens, window, sinks)
CASES = [
    (128, 32, 8, 16, [1, 2, 15, 16, 17, 31, 32, 33, 100, 1000, 0], 1, 0, 0),
    (128, 32, 8, 16, [5000], 1, 0, 0),                            # a split sequence, fixed chunks
    (128, 64, 8, 16, [3, 64, 700], 2, 0, 0),                      # 16 columns
    (128, 40, 8, 32, [1, 2, 3, 33, 900, 4000], 3, 0, 0),          # 15 columns, fewer tokens than queries
    (128, 16, 1, 64, [0, 1, 63, 64, 65, 3000], 1, 0, 0),          # G = 16, one kv head: eight step phases
    (128, 12, 3, 16, [40, 77, 2000], 1, 0, 0),                    # three kv heads
    (128, 7, 7, 16, [40, 77, 500], 2, 0, 0),                      # odd head counts
    (64, 8, 2, 16, [1, 31, 256, 777], 1, 0, 0),
    (64, 6, 2, 128, [1, 127, 129, 1000], 5, 0, 0),
    (256, 12, 4, 16, [1, 31, 33, 500, 0], 1, 0, 0),
    (256, 8, 1, 1024, [1023, 1025, 3000], 2, 0, 0),
    (128, 32, 8, 16, [1, 33, 100, 1000, 0], 1, 64, 4),
    (128, 32, 8, 16, [5, 66, 1027, 3000], 4, 100, 33),            # sinks past a step
    (128, 32, 8, 16, [5, 66, 1027, 3000], 2, 100, 0),
    (128, 32, 8, 16, [20, 900, 4000], 1, 1, 1),
    (128, 32, 8, 32, [900, 4000, 117], 3, 50, 500),               # more sinks than window
    (128, 8, 8, 64, [900, 4000], 16, 30, 17),
    (64, 16, 4, 16, [5, 64, 65, 300], 2, 37, 5),
    (256, 12, 4, 16, [5, 33, 66, 1027, 3000], 2, 100, 4),
]


@pytest.mark.parametrize("d,hq,hkv,page,lens,tq,window,sinks", CASES,
                         ids=[f"D{c[0]}-{c[1]}:{c[2]}-P{c[3]}-T{c[5]}-W{c[6]}-S{c[7]}" for c in CASES])
def test_attention_shapes(lib, d, hq, hkv, page, lens, tq, window, sinks):
    w = build(lens, hq, hkv, d, page, seed=sum(lens) + tq + window, num_queries=tq, window=window, sinks=sinks)
    cache = quantised(w)  # dead and hidden tokens are NaN groups (scale 255)
    log(f"kv4 D={d} {hq}:{hkv} P={page} lens={lens} Tq={tq} W={window} S={sinks}")
    check(run(lib, w, cache, window, sinks), ref(w, cache, window, sinks), "kv4")


@pytest.mark.parametrize("min_steps,blocks", [(1, 1), (1, 4), (7, 2), (1 << 20, 1)])
@pytest.mark.parametrize("fixed", [0, 1])
def test_attention_split_sweep(lib, min_steps, blocks, fixed):
    lib.set_option(lib.OPT_MIN_STEPS, min_steps)
    lib.set_option(lib.OPT_BLOCKS_PER_CU, blocks)
    lib.set_option(lib.OPT_FIXED_SPLIT, fixed)
    try:
        for tq, window, sinks in [(1, 0, 0), (4, 0, 0), (2, 45, 0), (4, 33, 70)]:
            w = build([33, 66, 97, 1027, 2050], 32, 8, 128, 16, seed=70 + tq + window, num_queries=tq, window=window, sinks=sinks)
            cache = quantised(w)
            log(f"sweep min_steps={min_steps} blocks={blocks} fixed={fixed} Tq={tq} W={window} S={sinks}")
            check(run(lib, w, cache, window, sinks), ref(w, cache, window, sinks), f"Tq={tq} W={window}")
    finally:
        lib.set_option(lib.OPT_MIN_STEPS, 0)
        lib.set_option(lib.OPT_BLOCKS_PER_CU, 1)
        lib.set_option(lib.OPT_FIXED_SPLIT, 1)


@pytest.mark.parametrize("batch,lo,hi", [(300, 1, 140), (700, 1, 64), (1100, 0, 40)])
def test_attention_many_sequences(lib, batch, lo, hi):
    rng = np.random.default_rng(batch)
    w = build(rng.integers(lo, hi, batch).tolist(), 8, 2, 128, 16, seed=batch)
    cache = quantised(w)
    log(f"kv4 batch={batch}")
    check(run(lib, w, cache), ref(w, cache), f"batch {batch}")


@pytest.mark.parametrize("scale", [-0.09, 0.0, 1.5])
def test_attention_scales(lib, scale):
    # a negative scale turns the order of the scores, zero makes them equal, a large one leaves one key
    w = build([1, 33, 700], 32, 8, 128, 16, seed=9, num_queries=2, window=300, sinks=3)
    cache = quantised(w)
    check(run(lib, w, cache, 300, 3, scale), ref(w, cache, 300, 3, scale), f"scale {scale}")


def test_attention_key_and_value_scales_far_apart(lib):
    # groups whose units differ by 2^40 within one row, values up to 2^60
    rng = np.random.default_rng(4)
    w = build([40, 300], 8, 2, 128, 16, seed=4, poison=False)
    kc, ks, vc, vs = quantised(w)
    ks = ks.copy()
    ks[:, :, 1] = rng.integers(80, 126, ks[:, :, 1].shape)
    vs = rng.integers(100, 130, vs.shape).astype(np.uint8)
    vs[:, :, 2] += 60
    cache = (kc, ks, vc, vs)
    got, want = run(lib, w, cache), ref(w, cache)
    group = want.reshape(*want.shape[:-1], 4, 32)
    size = np.abs(group).max(axis=-1, keepdims=True)
    assert (np.abs(got.reshape(group.shape) - group) <= 2.0 ** -8 * size).all()


def test_attention_dominant_key_returns_its_value(lib):
    w = build([2000], 32, 8, 128, 16, seed=10, poison=False)
    kc, ks, vc, vs = quantised(w)
    page, slot = int(w.block_table[0, 1234 // 16]), 1234 % 16
    ks[page, :, :, slot] = 140
    got, want = run(lib, w, (kc, ks, vc, vs)), ref(w, (kc, ks, vc, vs))
    check(got, want, "dominant")


def test_visible_nan_reaches_the_output_and_no_further(lib):
    w = build([40, 300], 8, 2, 128, 16, seed=11, poison=False)
    kc, ks, vc, vs = quantised(w)
    vs[int(w.block_table[0, 1]), 1, 3, 2] = 255     # value of token 18, kv head 1, d 96..127, of the first sequence
    got = run(lib, w, (kc, ks, vc, vs))
    bad = np.isnan(got)
    assert bad[0, :, 4:, 96:].all() and bad.sum() == bad[0, :, 4:, 96:].size


def test_attention_on_another_stream_and_in_a_graph(lib):
    import torch
    w = build([700, 33, 5000], 32, 8, 128, 16, seed=83, num_queries=2, window=256, sinks=20)
    cache = quantised(w)
    want = ref(w, cache, 256, 20)
    s = torch.cuda.Stream()
    check(run(lib, w, cache, 256, 20, stream=s), want, "own stream")
    q, dev = torch_bf16(w.q), [torch_any(t) for t in cache]
    table, lens = torch_any(w.block_table), torch_any(w.context_lens)
    out = torch.zeros_like(q)
    new = torch.randn((3, 2, 8, 128), device="cuda").bfloat16()
    lib.kv4_workspace_reserve(3, 32, 8, 128, 16, table.shape[1], stream=s)
    eager = [t.clone() for t in dev]
    lib.kv4_append(new, new, *eager, table, lens)
    eager_out = torch.zeros_like(q)
    lib.paged_decode_attention_kv4(q, *eager, table, lens, eager_out, float(w.scale), window=256, sinks=20)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        lib.kv4_append(new, new, *dev, table, lens)
        lib.paged_decode_attention_kv4(q, *dev, table, lens, out, float(w.scale), window=256, sinks=20)
    for rep in range(4):
        out.zero_()
        run(lib, w, cache)  # eager work of the same kernels in between
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager_out), rep
        assert all(torch.equal(a, b) for a, b in zip(dev, eager))


def test_capture_without_a_reserve_is_refused(lib):
    import torch
    w = build([5000], 32, 8, 128, 16, seed=84)
    q, dev = torch_bf16(w.q), [torch_any(t) for t in quantised(w)]
    table, lens, out = torch_any(w.block_table), torch_any(w.context_lens), torch.zeros_like(q)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    lib.release_workspaces()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        with pytest.raises(lib.PdaError, match="reserve"):
            lib.paged_decode_attention_kv4(q, *dev, table, lens, out, float(w.scale))
        out.zero_()
    torch.cuda.synchronize()


def test_pools_past_four_gigabytes(lib):
    import torch
    n, hkv, d, page = 300_000, 8, 256, 16  # codes: 4.9 GB a pool
    w = build([33, 700], 16, hkv, d, page, seed=12, poison=False)
    small = quantised(w)
    used = w.k_cache.shape[0]
    far = np.random.default_rng(1).choice(np.arange(n - 2000, n), used, replace=False)
    dev = []
    for t in small:
        big = torch.zeros((n, *t.shape[1:]), dtype=torch.uint8, device="cuda")
        big[torch.from_numpy(far).cuda()] = torch_any(t)
        dev.append(big)
    table = np.where(w.block_table >= 0, far[np.maximum(w.block_table, 0)], -1).astype(np.int32)
    q, out = torch_bf16(w.q), torch.empty(w.q.shape, dtype=torch.bfloat16, device="cuda")
    lib.paged_decode_attention_kv4(q, *dev, torch_any(table), torch_any(w.context_lens), out, float(w.scale))
    check(out.float().cpu().numpy().astype(np.float64), ref(w, small), "far pages")
    new = torch.randn((2, 3, hkv, d), device="cuda").bfloat16()
    back = [torch.empty_like(new) for _ in range(2)]
    lib.kv4_append(new, new, *dev, torch_any(table), torch_any(w.context_lens))
    lib.kv4_read(*back, *dev, torch_any(table), torch_any(w.context_lens))
    bits = new.view(torch.int16).cpu().numpy().view(np.uint16)
    want = C.kv4_values(*C.kv4_quantise(bits)).reshape(bits.shape)
    assert all(np.array_equal(b.float().cpu().numpy().astype(np.float64), want) for b in back)


def test_bad_page_ids_and_lengths_stay_inside(lib):
    # entries outside the pool and lengths outside the table are clamped: values unspecified, no fault
    import torch
    w = build([40, 300], 8, 2, 128, 16, seed=13, poison=False)
    w.block_table[0, 1] = 1 << 30
    w.block_table[1, 0] = -5
    w.context_lens = np.array([1 << 30, -3], dtype=np.int32)
    got = run(lib, w, quantised(w))
    assert (got[1] == 0).all()
    torch.cuda.synchronize()


def test_refusals(lib):
    import torch
    w = build([40, 300], 8, 2, 128, 16, seed=14)
    q, dev = torch_bf16(w.q), [torch_any(t) for t in quantised(w)]
    table, lens, out = torch_any(w.block_table), torch_any(w.context_lens), torch.zeros_like(torch_bf16(w.q))

    def call(q=q, cache=dev, table=table, lens=lens, out=out, scale=0.1, **kw):
        return lib.paged_decode_attention_kv4(q, *cache, table, lens, out, scale, **kw)

    with pytest.raises(ValueError, match="k_scales"):
        call(cache=[dev[0], dev[1][:, :1].contiguous(), *dev[2:]])
    with pytest.raises(TypeError, match="v_codes"):
        call(cache=[*dev[:2], dev[2].view(torch.int8), dev[3]])
    with pytest.raises(ValueError, match="contiguous"):
        call(q=torch.cat([q, q], dim=-1)[..., :128])
    with pytest.raises(ValueError, match="groups"):
        call(q=q[..., :64].contiguous(), out=out[..., :64].contiguous())
    with pytest.raises(lib.PdaError, match="window"):
        call(window=-1)
    with pytest.raises(lib.PdaError, match="num_sinks"):
        call(window=5, sinks=-1)
    with pytest.raises(lib.PdaError, match="scale"):
        call(scale=float("inf"))
    with pytest.raises(ValueError, match="k_new"):
        lib.kv4_append(q[:, 0], q[:, 0], *dev, table, lens)
    assert (out == 0).all()


def test_empty_batch(lib):
    import torch
    c, s = lib.kv4_cache(4, 16, 2, 128)
    q = torch.zeros((0, 1, 8, 128), dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros((0, 3), dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    lib.paged_decode_attention_kv4(q, c, s, c, s, table, lens, q, 0.1)
    kv = torch.zeros((0, 1, 2, 128), dtype=torch.bfloat16, device="cuda")
    lib.kv4_append(kv, kv, c, s, c, s, table, lens)
