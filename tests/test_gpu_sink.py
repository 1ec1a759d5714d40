"""GPU parity of the bf16 cache's attention with a sliding window and sinks, against the fp64 reference.

Same bar as the other variants: every output within one bf16 spacing of the
fp64 value.  What no query sees is NaN, and pages without any other token are
released (-1).
"""
import numpy as np
import pytest

import oracle
from _cache import build, torch_any, torch_bf16
from _gpu import check, log
from oracle import cache as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


def device(w):
    return torch_bf16(w.q), torch_bf16(w.k_cache), torch_bf16(w.v_cache), torch_any(w.block_table), torch_any(w.context_lens)


def run(lib, w, window, sinks, stream=None):
    import torch
    q, k, v, bt, lens = device(w)
    out = torch.full(tuple(q.shape), float("nan"), dtype=torch.bfloat16, device="cuda")
    lib.paged_decode_attention_sink(q, k, v, bt, lens, out, float(w.scale), window=window, sinks=sinks, stream=stream)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


def ref(w, window, sinks):
    return C.attend(w.q, oracle.bf16_to_f64(w.k_cache), oracle.bf16_to_f64(w.v_cache), w.block_table, w.context_lens, w.scale,
                    window, sinks)


# (head_dim, Hq, Hkv, page, lengths, query tokens, window, sinks)
CASES = [
    (128, 32, 8, 16, [0, 1, 4, 5, 33, 68, 69, 100, 1000], 1, 64, 4),
    (128, 32, 8, 16, [5, 66, 1027, 3000], 4, 100, 33),       # sinks past a step
    (128, 32, 8, 16, [20, 900, 4000], 1, 1, 1),
    (128, 32, 8, 16, [900, 4000, 117], 3, 50, 500),          # more sinks than window
    (128, 16, 1, 32, [7, 700, 4099], 1, 513, 15),            # eight step phases
    (128, 16, 1, 32, [7, 700, 4099], 1, 513, 17),
    (128, 8, 8, 16, [20, 900], 16, 30, 16),                  # sinks end with a page
    (128, 8, 8, 1024, [1023, 1025, 3000], 1, 1500, 9),
    (64, 16, 4, 4, [5, 64, 65, 300], 2, 37, 6),              # pages below 16 tokens
    (64, 12, 4, 1, [2, 40, 333], 3, 9, 2),
    (64, 4, 2, 64, [129, 4000, 64], 8, 2000, 77),
    (256, 12, 4, 16, [5, 33, 66, 1027, 3000], 2, 100, 4),
    (256, 4, 4, 4, [5, 64, 65, 300], 3, 37, 40),
    (128, 40, 8, 32, [20001], 1, 1024, 4),                   # one long sequence: fixed chunks
    (128, 32, 8, 16, [64, 100, 4000], 2, 1 << 30, 4),        # a window past every length
    (128, 32, 8, 16, [64, 100, 4000], 2, 32, 1 << 30),       # sinks past every length
]


@pytest.mark.parametrize("d,hq,hkv,page,lens,tq,window,sinks", CASES,
                         ids=[f"D{c[0]}-{c[1]}:{c[2]}-P{c[3]}-T{c[5]}-W{c[6]}-S{c[7]}" for c in CASES])
def test_sink_shapes(lib, d, hq, hkv, page, lens, tq, window, sinks):
    w = build(lens, hq, hkv, d, page, seed=sum(lens) + 13 * tq + window, num_queries=tq, window=window, sinks=sinks)
    log(f"sink D={d} {hq}:{hkv} P={page} lens={lens} Tq={tq} W={window} S={sinks}")
    check(run(lib, w, window, sinks), ref(w, window, sinks), "sink")


@pytest.mark.parametrize("min_steps,blocks", [(1, 1), (1, 4), (7, 2), (1 << 20, 1)])
@pytest.mark.parametrize("fixed", [0, 1])
def test_sink_split_sweep(lib, min_steps, blocks, fixed):
    lib.set_option(lib.OPT_MIN_STEPS, min_steps)
    lib.set_option(lib.OPT_BLOCKS_PER_CU, blocks)
    lib.set_option(lib.OPT_FIXED_SPLIT, fixed)
    try:
        for tq, window, sinks in [(1, 45, 1), (2, 45, 40), (4, 33, 70)]:
            w = build([33, 66, 97, 1027, 2050], 32, 8, 128, 16, seed=70 + tq + window, num_queries=tq, window=window, sinks=sinks)
            log(f"sweep min_steps={min_steps} blocks={blocks} fixed={fixed} Tq={tq} W={window} S={sinks}")
            check(run(lib, w, window, sinks), ref(w, window, sinks), f"Tq={tq} W={window} S={sinks}")
    finally:
        lib.set_option(lib.OPT_MIN_STEPS, 0)
        lib.set_option(lib.OPT_BLOCKS_PER_CU, 1)
        lib.set_option(lib.OPT_FIXED_SPLIT, 1)


def test_a_batch_of_many_sequences(lib):
    rng = np.random.default_rng(3)
    w = build(rng.integers(0, 150, 700).tolist(), 8, 2, 64, 16, seed=3, window=40, sinks=5)
    check(run(lib, w, 40, 5), ref(w, 40, 5), "700 sequences")


def test_no_sinks_and_no_window_are_the_other_calls_bitwise(lib):
    import torch
    w = build([33, 700, 3000], 32, 8, 128, 16, seed=21, num_queries=2, poison=False)
    q, k, v, bt, lens = device(w)
    for window in (0, 100):
        out = torch.empty_like(q)
        lib.paged_decode_attention_ext(q, k, v, bt, lens, out, float(w.scale), window=window)
        want = out.float().cpu().numpy().astype(np.float64)
        assert np.array_equal(run(lib, w, window, 0), want)
    assert np.array_equal(run(lib, w, 0, 4), run(lib, w, 0, 0))


def test_other_options_do_not_change_the_call(lib):
    w = build([33, 700, 3000], 32, 8, 128, 16, seed=22, window=100, sinks=4)
    want = run(lib, w, 100, 4)
    for option, value in ((lib.OPT_COMPUTE_PATH, 1), (lib.OPT_FUSED_MERGE, 2)):
        lib.set_option(option, value)
        try:
            assert np.array_equal(run(lib, w, 100, 4), want)
        finally:
            lib.set_option(option, 0)


def test_graph_replays_on_another_stream(lib):
    import torch
    w = build([700, 33, 5000], 32, 8, 128, 16, seed=83, num_queries=4, window=256, sinks=20)
    q, k, v, bt, lens = device(w)
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    lib.workspace_reserve(3, 32, 8, 128, 16, w.max_pages, stream=s)
    want = run(lib, w, 256, 20)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        lib.paged_decode_attention_sink(q, k, v, bt, lens, out, float(w.scale), window=256, sinks=20)
    for rep in range(4):
        out.zero_()
        run(lib, w, 100, 3)
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.float().cpu().numpy().astype(np.float64), want), rep
    check(want, ref(w, 256, 20), "graph")


def test_refusals(lib):
    import torch
    w = build([40], 8, 2, 128, 16, seed=23)
    q, k, v, bt, lens = device(w)
    out = torch.zeros_like(q)
    with pytest.raises(lib.PdaError, match="num_sinks"):
        lib.paged_decode_attention_sink(q, k, v, bt, lens, out, 0.1, window=5, sinks=-1)
    with pytest.raises(lib.PdaError, match="window"):
        lib.paged_decode_attention_sink(q, k, v, bt, lens, out, 0.1, window=-5, sinks=1)
    with pytest.raises(ValueError, match="out"):
        lib.paged_decode_attention_sink(q, k, v, bt, lens, out[:, 0], 0.1, window=5, sinks=1)
    assert (out == 0).all()
