"""The cache operators at the ends of what their arguments can hold, against the fp64 reference."""
import numpy as np
import pytest

import oracle
from _cache import build, torch_any, torch_bf16
from _gpu import check, log
from oracle import cache as C
from test_gpu_cache_limits import compare, partly_seen
from test_gpu_kv4 import quantised
from test_gpu_kv4 import run as run_kv4
from test_gpu_sink import run as run_sink

pytestmark = pytest.mark.gpu

INT_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


def run_ext(lib, w, window):
    import torch
    q = torch_bf16(w.q)
    out = torch.full(tuple(q.shape), float("nan"), dtype=torch.bfloat16, device="cuda")
    lib.paged_decode_attention_ext(q, torch_bf16(w.k_cache), torch_bf16(w.v_cache), torch_any(w.block_table),
                                   torch_any(w.context_lens), out, float(w.scale), window=window)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


# ------------------------------------------------------------ window and sinks
# (head_dim, Hq, Hkv, page, lengths, query tokens): sequences shorter than their queries, idle slots alone and
# beside others
SHORT = [(128, 32, 8, 16, [0, 1, 2, 5, 33, 700], 4), (128, 8, 8, 16, [0, 13, 15, 3000], 16), (64, 6, 2, 32, [0, 0, 0], 5),
         (256, 12, 4, 16, [0, 1, 64, 500], 3), (64, 4, 2, 64, [1], 8)]


@pytest.mark.parametrize("fixed", [0, 1])
@pytest.mark.parametrize("window", [INT_MAX, INT_MAX - 1, INT_MAX - 14, 1 << 30])
@pytest.mark.parametrize("d,hq,hkv,page,lens,tq", SHORT, ids=[f"D{c[0]}-{c[1]}:{c[2]}-T{c[5]}" for c in SHORT])
def test_a_window_past_every_position_hides_nothing(lib, d, hq, hkv, page, lens, tq, window, fixed):
    w = build(lens, hq, hkv, d, page, seed=sum(lens) + tq, num_queries=tq)
    cache = quantised(w)
    log(f"window {window} D={d} {hq}:{hkv} lens={lens} Tq={tq} fixed={fixed}")
    lib.set_option(lib.OPT_FIXED_SPLIT, fixed)
    try:
        bf16 = C.attend(w.q, oracle.bf16_to_f64(w.k_cache), oracle.bf16_to_f64(w.v_cache), w.block_table, w.context_lens, w.scale)
        check(run_ext(lib, w, window), bf16, "ext")
        kv4 = C.attend(w.q, C.kv4_tokens(*cache[:2]), C.kv4_tokens(*cache[2:]), w.block_table, w.context_lens, w.scale)
        for sinks in (0, 4, INT_MAX):
            check(run_sink(lib, w, window, sinks), bf16, f"sink {sinks}")
            check(run_kv4(lib, w, cache, window, sinks), kv4, f"kv4 {sinks}")
    finally:
        lib.set_option(lib.OPT_FIXED_SPLIT, 1)


def test_sinks_past_every_position_leave_nothing_hidden(lib):
    w = build([0, 3, 700], 32, 8, 128, 16, seed=31, num_queries=4)
    want = C.attend(w.q, oracle.bf16_to_f64(w.k_cache), oracle.bf16_to_f64(w.v_cache), w.block_table, w.context_lens, w.scale)
    check(run_sink(lib, w, 7, INT_MAX), want, "sink")


# ------------------------------------------------------- tokens without a page
# (head_dim, kv heads, page, tokens, length): single tokens and runs of eight
NOWHERE = [(128, 8, 16, 1, 40), (64, 2, 16, 5, 40), (256, 2, 32, 40, 100), (128, 3, 16, 33, 70)]


@pytest.mark.parametrize("entry", [-1, -7, 2 ** 31 - 1, None])  # None: the first number past the pool
@pytest.mark.parametrize("d,hkv,page,tokens,length", NOWHERE)
def test_kv4_tokens_without_a_page_go_nowhere(lib, d, hkv, page, tokens, length, entry):
    import torch
    rng = np.random.default_rng(d + tokens)
    pages = 30
    codes = rng.integers(0, 256, (2, pages, hkv, d // 32, page, 16), np.uint8)
    scales = rng.integers(0, 255, (2, pages, hkv, d // 32, page), np.uint8)
    used = -(-length // page)
    table = np.full((2, used), -1, np.int32)
    table[0] = rng.choice(pages - 1, used, replace=False)  # the last page is nobody's
    table[1] = pages if entry is None else entry            # the second sequence has no page at all
    table[0, -2] = table[1, 0]                              # the first lacks its last page but one
    lens = np.array([length, length - 1], np.int32)
    new = [rng.integers(0, 0x7F80, (2, tokens, hkv, d)).astype(np.uint16) for _ in range(2)]
    dev = [torch_any(x) for x in (codes[0], scales[0], codes[1], scales[1])]
    bt, cl = torch_any(table), torch_any(lens)
    log(f"kv4 without a page D={d} P={page} T={tokens} entry={entry}")
    lib.kv4_append(torch_bf16(new[0]), torch_bf16(new[1]), *dev, bt, cl)
    back = [torch.full((2, tokens, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib.kv4_read(*back, *dev, bt, cl)
    torch.cuda.synchronize()
    t = lens[0] - tokens + np.arange(tokens)  # the first sequence's tokens, those with a page
    here = [j for j in range(tokens) if t[j] >= 0 and t[j] // page != used - 2]
    for i in range(2):
        c, s = codes[i].copy(), scales[i].copy()
        for j in here:
            qc, qs = C.kv4_quantise(new[i][0, j])
            c[table[0, t[j] // page], :, :, t[j] % page] = qc
            s[table[0, t[j] // page], :, :, t[j] % page] = qs
        assert np.array_equal(dev[2 * i].cpu().numpy(), c) and np.array_equal(dev[2 * i + 1].cpu().numpy(), s)
        got = back[i].float().cpu().numpy()
        assert (got[1] == 0).all() and (np.delete(got[0], here, axis=0) == 0).all()
        want = C.kv4_values(*C.kv4_quantise(new[i][0, here])).reshape(len(here), hkv, d)
        assert np.array_equal(got[0, here], want.astype(np.float32))


@pytest.mark.parametrize("entry", [-1, 2 ** 31 - 1, None])
@pytest.mark.parametrize("d,hkv,page,tokens,length", NOWHERE + [(128, 2, 1, 7, 20), (64, 4, 4, 1, 9)])
def test_bf16_tokens_without_a_page_go_nowhere(lib, d, hkv, page, tokens, length, entry):
    import torch
    rng = np.random.default_rng(d + tokens)
    used = -(-length // page)
    pages = 3 * used
    pools = rng.integers(0, 0x7F80, (2, pages, page, hkv, d)).astype(np.uint16)
    table = np.full((2, used), -1, np.int32)
    table[0] = rng.choice(pages - 1, used, replace=False)
    table[1] = pages if entry is None else entry
    table[0, -2] = table[1, 0]
    lens = np.array([length, length - 1], np.int32)
    new = rng.integers(0, 0x7F80, (2, 2, tokens, hkv, d)).astype(np.uint16)
    dev = [torch_bf16(p) for p in pools]
    log(f"bf16 without a page D={d} P={page} T={tokens} entry={entry}")
    lib.kv_append_n(torch_bf16(new[0]), torch_bf16(new[1]), *dev, torch_any(table), torch_any(lens))
    torch.cuda.synchronize()
    for i in range(2):
        want = pools[i].copy()
        for j in range(tokens):
            t = length - tokens + j
            if t >= 0 and t // page != used - 2:
                want[table[0, t // page], t % page] = new[i][0, j]
        assert np.array_equal(dev[i].view(torch.int16).cpu().numpy().view(np.uint16), want)


# (batch, hidden, Hq, Hkv, D, q/k norm): without a norm the projection's workgroups finish the prelude, with one
# a second kernel does
@pytest.mark.parametrize("entry", [-1, None])
@pytest.mark.parametrize("b,hidden,hq,hkv,d,norm", [
    (1, 2560, 32, 8, 128, False), (6, 512, 8, 2, 128, True), (8, 4096, 32, 2, 128, False), (64, 1024, 8, 2, 128, False),
    (100, 512, 4, 2, 128, True), (256, 512, 8, 2, 128, False), (16, 768, 12, 4, 256, True), (16, 768, 12, 4, 256, False),
    (3, 1024, 4, 2, 64, True)])
def test_a_prelude_appends_nothing_without_a_page(lib, b, hidden, hq, hkv, d, norm, entry):
    import torch
    rng = np.random.default_rng(b + hidden)
    plan = lib.prelude_plan(lib.prelude_dims(b, hidden, hq, hkv, d, d, False, 1e5, 1e-6), norm)
    assert bool(plan.fused) == (not norm)
    page, used = 16, 3
    lens = rng.integers(1, page * used + 1, b).astype(np.int32)
    pages = used * b + 5
    table = rng.permutation(pages - 1)[:used * b].reshape(b, used).astype(np.int32)  # the last page is nobody's
    lost = [r for r in range(b) if r % 2 == 0]
    for r in lost:
        table[r, (lens[r] - 1) // page] = pages if entry is None else entry
    pools = [rng.integers(0, 0x7F80, (pages, page, hkv, d)).astype(np.uint16) for _ in range(2)]
    x = torch.randn((b, hidden), device="cuda").bfloat16()
    wp = lib.pack_weights((torch.randn(((hq + 2 * hkv) * d, hidden), device="cuda") * hidden ** -0.5).bfloat16())
    norms = dict(q_norm=torch.ones(d, dtype=torch.bfloat16, device="cuda"),
                 k_norm=torch.ones(d, dtype=torch.bfloat16, device="cuda")) if norm else {}
    shape = dict(num_q_heads=hq, num_kv_heads=hkv, head_dim=d, rope_theta=1e5, **norms)
    q, q2 = (torch.empty((b, hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.empty((b, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cl, dev = torch_any(lens), [torch_bf16(p) for p in pools]
    log(f"prelude without a page B={b} {hq}:{hkv} D={d} norm={norm} entry={entry}")
    lib.attention_prelude(x, wp, cl, q, k, v, **shape)
    lib.attention_prelude_append(x, wp, cl, q2, *dev, torch_any(table), **shape)
    torch.cuda.synchronize()
    assert torch.equal(q, q2)
    for pool, new, got in zip(pools, (k, v), dev):
        want, rows = pool.copy(), new.view(torch.int16).cpu().numpy().view(np.uint16)
        for r in range(b):
            if r not in lost:
                t = lens[r] - 1
                want[table[r, t // page], t % page] = rows[r]
        assert np.array_equal(got.view(torch.int16).cpu().numpy().view(np.uint16), want)


# --------------------------------------------------- the checks of a debugging run
VALIDATED = """
import sys, torch
sys.path.insert(0, '.')
from paper_2606_07665_amd import binding as B
dev = dict(dtype=torch.int32, device='cuda')
N, P, M, HQ, HKV, D, W, S, T = 80, 16, 40, 8, 2, 128, 50, 20, 3
table, lens = torch.arange(80, **dev).reshape(2, M), torch.tensor([400, 600], **dev)
ref = (torch.arange(80, device='cuda') < 25).int() + ((torch.arange(80, device='cuda') >= 40) & (torch.arange(80, device='cuda') < 78)).int()
new = torch.tensor([403, 603], **dev)
t2, r2, src, dst, info = torch.empty_like(table), torch.empty_like(ref), torch.empty(2, **dev), torch.empty(2, **dev), torch.empty(2, **dev)
B.pages_update(table, lens, None, new, ref, t2, r2, src, dst, info, page_size=P, window=W, sinks=S, num_queries=T)
held = (t2 >= 0).sum(dim=1).tolist()
assert held[0] < 10 and held[1] < 10, held          # most pages are released
k, v = (torch.randn((N, P, HKV, D), device='cuda').bfloat16() for _ in range(2))
c4 = [*B.kv4_cache(N, P, HKV, D), *B.kv4_cache(N, P, HKV, D)]
q = torch.randn((2, T, HQ, D), device='cuda').bfloat16()
out, kn = torch.zeros_like(q), torch.randn((2, T, HKV, D), device='cuda').bfloat16()
calls = dict(
    sink=lambda t: B.paged_decode_attention_sink(q, k, v, t, new, out, 0.1, window=W, sinks=S),
    kv4=lambda t: B.paged_decode_attention_kv4(q, *c4, t, new, out, 0.1, window=W, sinks=S),
    append=lambda t: B.kv4_append(kn, kn, *c4, t, new),
    read=lambda t: B.kv4_read(kn, kn.clone(), *c4, t, new),
    bf16=lambda t: B.kv_append_n(kn, kn, k, v, t, new))
ext = lambda t: B.paged_decode_attention_ext(q, k, v, t, new, out, 0.1, window=W)

def refused(call, t):
    try:
        call(t)
        return ''
    except B.PdaError as e:
        return str(e)

for name, call in calls.items():
    assert not refused(call, t2), name
    last = t2.clone()
    last[1, 602 // P] = -1
    assert 'block_table[1][37]' in refused(call, last), name
    bad = t2.clone()
    bad[0, 1] = N + 3                                # the sinks' second page: attention sees it, the others do not
    assert ('block_table[0][1]' in refused(call, bad)) == (name in ('sink', 'kv4')), name
gone = t2.clone()
gone[:, :2] = -1
assert not refused(ext, gone) and 'block_table[0][0]' in refused(calls['sink'], gone)
first = (403 - T + 1 - W) // P                       # the window's first page, and the one before it
edge = t2.clone()
edge[0, first - 1] = N
assert not refused(ext, edge) and not refused(calls['kv4'], edge)
edge[0, first] = N
assert f'block_table[0][{first}]' in refused(ext, edge) and f'block_table[0][{first}]' in refused(calls['kv4'], edge)
plain = lambda t: B.paged_decode_attention_ext(q, k, v, t, new, out, 0.1)
assert 'block_table' in refused(plain, t2)           # without a window every page is seen
print('AS IT SHOULD')
"""


def test_a_debugging_run_checks_the_pages_that_a_call_touches():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", VALIDATED], cwd=root, env=dict(os.environ, PDA_DEBUG_VALIDATE="1"),
                       capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "AS IT SHOULD" in r.stdout, r.stdout + r.stderr[-2000:]


# ------------------------------------------------------------ the largest values
# Scores are 0 but for a few tokens at 7.9 in log2 units, which a softmax whose reference lags by up to 8 takes
# as probabilities of 2^7.9.  "one": such a token has values up to the format's largest, 1.5 * 2^127.  "after":
# 128 tokens with a score of 0 have values up to 2^126.6, behind one such token of each wave: their sum stays in
# fp32 relative to the largest probability, which holds only in waves that see both.
@pytest.mark.parametrize("kind,min_steps", [("one", 0), ("one", 1 << 20), ("after", 1 << 20)])  # waves of a step or two, of many
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("d,hq,hkv,batch", [(128, 8, 2, 3), (64, 4, 4, 3), (256, 4, 1, 2), (128, 16, 8, 10)])
def test_kv4_values_near_the_top_of_the_range(lib, d, hq, hkv, batch, kind, sign, min_steps):
    rng = np.random.default_rng(d + batch)
    n, page = 1500, 16
    w = build([n] * batch, hq, hkv, d, page, seed=d, poison=False)
    kc, ks, vc, vs = (t.copy() for t in quantised(w))
    kc[:], ks[:], vc[:], vs[:] = 0, 127, 0, 100
    w.q[:] = 0
    w.q[..., 0] = 0x3F80  # 1.0: a score is element 0 of the key
    scale = sign * 7.9 / 6 * np.log(2.0)

    def slot(b, t):
        return int(w.block_table[b, t // page]), t % page

    for b in range(batch):
        for t in ([700] if kind == "one" else [32 * s + 5 for s in range(4, 8)]):
            at, s = slot(b, t)
            kc[at, :, 0, s, 0] = 0x07 if sign > 0 else 0x0F  # 6 or -6
        for t in ([700] if kind == "one" else range(256, 384)):
            at, s = slot(b, t)
            vs[at, :, :, s] = 252 if kind == "one" else 251
            vc[at, :, :, s] = rng.integers(0, 256, vc[at, :, :, s].shape)
    cache = (kc, ks, vc, vs)
    lib.set_option(lib.OPT_MIN_STEPS, min_steps)
    lib.set_option(lib.OPT_FIXED_SPLIT, int(min_steps == 0))
    try:
        log(f"large values D={d} {hq}:{hkv} B={batch} {kind} sign={sign} min_steps={min_steps}")
        got = run_kv4(lib, w, cache, scale=scale)
        w.k_cache, w.v_cache = (np.asarray(bits_of(C.kv4_tokens(*cache[2 * i:2 * i + 2]))) for i in range(2))
        w.scale = scale
        bf16 = run_sink(lib, w, 0, 0)
    finally:
        lib.set_option(lib.OPT_MIN_STEPS, 0)
        lib.set_option(lib.OPT_FIXED_SPLIT, 1)
    want = C.attend(w.q, C.kv4_tokens(kc, ks), C.kv4_tokens(vc, vs), w.block_table, w.context_lens, scale)
    assert np.isfinite(bf16).all() and np.isfinite(got).all()
    # (sums of large values of both signs: fp32's error relative to the largest, beside half a bf16 spacing)
    most = np.abs(want).max()
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -15 * most).all()


def bits_of(x):
    """float64 values that bf16 holds exactly, as its bits."""
    f = x.astype(np.float32)
    assert np.array_equal(f.astype(np.float64), x)
    return (f.view(np.uint32) >> 16).astype(np.uint16)


# -------------------------------------------------------- a scale of zero
@pytest.mark.parametrize("scale", [0.0, -0.0])
@pytest.mark.parametrize("d,hq,hkv,lens,tq", [(128, 32, 8, [700, 33, 0], 1), (64, 8, 4, [100, 5000], 3), (256, 12, 4, [3, 400], 2)])
def test_kv4_queries_that_are_not_finite(lib, d, hq, hkv, lens, tq, scale):
    w = build(lens, hq, hkv, d, 16, seed=d + tq, num_queries=tq)
    cache = quantised(w)
    rng = np.random.default_rng(d)
    rows = [(b, j, int(h)) for b in range(len(lens)) for j in range(tq) for h in rng.choice(hq, 3, replace=False)]
    for i, (b, j, h) in enumerate(rows):
        w.q[b, j, h, (37 * i + 1) % d] = (0x7FC0, 0x7F80, 0xFF80, 0xFFC1)[i % 4]
    with np.errstate(invalid="ignore"):
        want = C.attend(w.q, C.kv4_tokens(*cache[:2]), C.kv4_tokens(*cache[2:]), w.block_table, w.context_lens, scale)
    log(f"queries not finite D={d} {hq}:{hkv} T={tq} scale={scale}")
    compare(run_kv4(lib, w, cache, scale=scale), want, f"scale {scale}")


# ------------------------------------------------------ sinks without a window
@pytest.mark.parametrize("pick", [0, -1, None])
@pytest.mark.parametrize("d,hq,hkv,page,lens,tq", [(128, 32, 8, 16, [300, 7, 2, 4000], 4), (64, 4, 2, 64, [129, 3], 8),
                                                   (256, 12, 4, 4, [100, 33], 3), (128, 8, 8, 1, [70, 15], 16)])
def test_bf16_values_reach_only_the_queries_that_see_them_without_a_window(lib, d, hq, hkv, page, lens, tq, pick):
    w = build(lens, hq, hkv, d, page, seed=sum(lens), num_queries=tq)
    for b, n in enumerate(lens):
        part = partly_seen(n, tq, 0, 4)
        for i, t in enumerate(part if pick is None else part[pick:][:1]):
            row = w.v_cache[int(w.block_table[b, t // page]), t % page]
            row[:, (7 * b + 11 * i + np.arange(hkv)) % d] = (0x7FC0, 0x7F80, 0xFF80)[(b + i) % 3]
    want = C.attend(w.q, oracle.bf16_to_f64(w.k_cache), oracle.bf16_to_f64(w.v_cache), w.block_table, w.context_lens, w.scale)
    log(f"bf16 partly seen, no window D={d} {hq}:{hkv} lens={lens} {pick}")
    compare(run_sink(lib, w, 0, 4), want, "sink")


@pytest.mark.parametrize("option", ["OPT_COMPUTE_PATH", "OPT_FUSED_MERGE"])
def test_options_leave_sinks_without_a_window_alone(lib, option):
    w = build([33, 700, 3000], 32, 8, 128, 16, seed=22, num_queries=2)
    want = run_sink(lib, w, 0, 4)
    lib.set_option(getattr(lib, option), 1)
    try:
        assert np.array_equal(run_sink(lib, w, 0, 4), want)
    finally:
        lib.set_option(getattr(lib, option), 0)


# ----------------------------------------------- numbers past 32 bits
@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32 + 16, -2 ** 32 + 16, 2 ** 64])
def test_numbers_past_32_bits_are_refused(lib, big):
    import torch
    w = build([100, 700], 8, 2, 128, 16, seed=1, poison=False)
    q, k, v = torch_bf16(w.q), torch_bf16(w.k_cache), torch_bf16(w.v_cache)
    table, lens, cache = torch_any(w.block_table), torch_any(w.context_lens), [torch_any(t) for t in quantised(w)]
    out = torch.zeros_like(q)
    for kw in (dict(window=big), dict(window=5, sinks=big)):
        name = "sinks" if "sinks" in kw else "window"
        with pytest.raises(ValueError, match=name):
            lib.paged_decode_attention_kv4(q, *cache, table, lens, out, 0.1, **kw)
        with pytest.raises(ValueError, match=name):
            lib.paged_decode_attention_sink(q, k, v, table, lens, out, 0.1, **kw)
    with pytest.raises(ValueError, match="window"):
        lib.paged_decode_attention_ext(q, k, v, table, lens, out, 0.1, window=big)
    n, dev = w.k_cache.shape[0], dict(dtype=torch.int32, device="cuda")
    ref = torch.ones(n, **dev)
    outs = [torch.full(s, 77, **dev) for s in (tuple(table.shape), (n,), (2,), (2,), (2,))]
    for kw in (dict(page_size=big), dict(page_size=16, window=big), dict(page_size=16, window=9, sinks=big),
               dict(page_size=16, num_queries=big)):
        with pytest.raises(ValueError, match="32-bit"):
            lib.pages_update(table, lens, None, lens, ref, *outs, **kw)
    outs = [torch.full(s, 77, **dev) for s in (tuple(table.shape), (n,), (n,), (n,), (n,), (2,))]
    with pytest.raises(ValueError, match="32-bit"):
        lib.pages_compact(table, lens, ref, *outs, page_size=big)
    torch.cuda.synchronize()
    assert (out == 0).all() and all((o == 77).all() for o in outs)


# ---------------------------------------- each side of the 4-bit call's forms
# (head_dim, Hq, Hkv, batch): three, or at head size 256 two, workgroups of 4 waves a CU up to the first batch of
# each pair, one of 12 (8) waves from the second on; then 12 and 8 waves, 8 and 4
@pytest.mark.parametrize("d,hq,hkv,batch", [(128, 4, 4, 2154), (128, 4, 4, 2155), (64, 4, 2, 4202), (64, 4, 2, 4203),
                                            (256, 2, 1, 1471), (256, 2, 1, 1472), (128, 4, 2, 6463), (128, 4, 2, 6464),
                                            (256, 2, 2, 2943), (256, 2, 2, 2944)])
def test_kv4_on_each_side_of_its_workgroups(lib, d, hq, hkv, batch):
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, 6, batch)
    lens[batch // 2] = 1500
    w = build(lens.tolist(), hq, hkv, d, 16, seed=batch)
    cache = quantised(w)
    want = C.attend(w.q, C.kv4_tokens(*cache[:2]), C.kv4_tokens(*cache[2:]), w.block_table, w.context_lens, w.scale)
    log(f"kv4 workgroups D={d} {hq}:{hkv} B={batch}")
    check(run_kv4(lib, w, cache), want, "workgroups")


# (Hq, Hkv, query tokens): 8 and 9, 10 columns: up to four kv heads a workgroup, up to two
@pytest.mark.parametrize("hq,hkv,tq", [(32, 8, 2), (24, 8, 3), (40, 8, 2), (16, 4, 2), (12, 4, 3)])
@pytest.mark.parametrize("longest", [4000, 9000])
def test_kv4_on_each_side_of_eight_columns(lib, hq, hkv, tq, longest):
    rng = np.random.default_rng(hq + tq)
    lens = rng.integers(0, 100, 64)
    lens[20] = longest
    w = build(lens.tolist(), hq, hkv, 128, 16, seed=hq + tq, num_queries=tq)
    cache = quantised(w)
    want = C.attend(w.q, C.kv4_tokens(*cache[:2]), C.kv4_tokens(*cache[2:]), w.block_table, w.context_lens, w.scale)
    log(f"kv4 columns {hq}:{hkv} T={tq} longest={longest}")
    check(run_kv4(lib, w, cache), want, "columns")
