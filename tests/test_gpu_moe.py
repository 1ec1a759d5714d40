"""GPU parity of routing and of the experts' products against the fp64 oracle."""
import numpy as np
import pytest
import torch

from _ffn import HALF, F32, TINY, activation_error, chain, check, f64, gpu, sum_error, values
from oracle import ffn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


# ------------------------------------------------------------------- routing
def route(lib, logits, top_k, **kw):
    t = logits.shape[0]
    ids = torch.full((t, top_k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((t, top_k), float("nan"), dtype=torch.float32, device="cuda")
    lib.moe_route(logits, ids, w, **kw)
    torch.cuda.synchronize()
    return ids.cpu().numpy(), f64(w)


def check_route(lib, logits, top_k, select_bias=None, **kw):
    got_ids, got_w = route(lib, gpu(logits), top_k, select_bias=gpu(select_bias), **kw)
    ids, w = ffn.moe_route(f64(logits), top_k, select_bias=None if select_bias is None else f64(select_bias), **kw)
    assert np.array_equal(got_ids, ids)
    # worked out in fp64, rounded to fp32 once
    assert (np.abs(got_w - w) <= 1.01 * F32 * np.abs(w) + 2.0 ** -149).all(), np.abs(got_w - w).max()


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("t,e,k", [(1, 1, 1), (1, 8, 2), (5, 60, 4), (3, 64, 8), (7, 65, 16), (33, 128, 8), (4, 200, 6),
                                   (64, 256, 8), (2, 511, 1), (3, 1024, 16), (1030, 16, 16)])
def test_route(lib, scoring, renormalise, bias, t, e, k):
    g = torch.Generator().manual_seed(t + e + k)
    check_route(lib, torch.randn(t, e, generator=g) * 2, k, torch.randn(e, generator=g) * 0.1 if bias else None,
                scoring=scoring, renormalise=renormalise, scale=2.5)


@pytest.mark.parametrize("bias", [False, True])
def test_route_ties_go_to_the_lowest(lib, bias):
    g = torch.Generator().manual_seed(1)
    logits = torch.randint(-2, 3, (64, 200), generator=g).float()
    logits[3] = 0.0
    logits[4, 7], logits[4, 150] = -0.0, 0.0
    # quarters: sigmoid or softmax scores tie where logits do, and the bias is one number
    check_route(lib, logits, 16, torch.full((200,), 0.25) if bias else None)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
def test_route_masks_infinities_and_nan(lib, scoring, bias):
    inf, nan = float("inf"), float("nan")
    rows = [[-inf] * 6, [nan] * 6, [-inf, 1.0, -inf, nan, 2.0, -inf], [inf, 0.0, inf, -inf, nan, 3.0],
            [3.4e38, -3.4e38, 0.0, 3.4e38, 1.0, -inf], [-3.4e38] * 6, [1e-40, -1e-40, 0.0, -0.0, nan, inf], [88.0, 89.0, -200.0, 700.0, 710.0, -745.0]]
    for renormalise in (True, False):
        check_route(lib, torch.tensor(rows), 5, torch.linspace(-0.2, 0.2, 6) if bias else None, scoring=scoring,
                    renormalise=renormalise)


def test_route_reads_a_wider_product_in_place(lib):
    g = torch.Generator().manual_seed(2)
    wide = torch.randn(9, 80, generator=g)
    wide[:, 60:] = float("nan")  # what lies past the experts is not looked at
    ids, w = route(lib, gpu(wide)[:, :60], 4)
    want_ids, want_w = ffn.moe_route(f64(wide[:, :60]), 4)
    assert np.array_equal(ids, want_ids) and np.allclose(w, want_w, rtol=1e-6)
    one = route(lib, gpu(wide)[:1, :60], 4)
    assert np.array_equal(one[0], want_ids[:1])


def test_route_leaves_the_rest_alone(lib):
    ids = torch.full((40,), -7, dtype=torch.int32, device="cuda")
    w = torch.full((40,), -7.0, device="cuda")
    lib.moe_route(torch.randn(5, 32, device="cuda"), ids[8:28].view(5, 4), w[8:28].view(5, 4))
    torch.cuda.synchronize()
    for t in (ids, w):
        assert (t[:8] == -7).all() and (t[28:] == -7).all() and (t[8:28] != -7).all()


def test_route_of_no_tokens(lib):
    ids, w = route(lib, torch.empty((0, 8), device="cuda"), 2)
    assert ids.shape == (0, 2)


# ------------------------------------------------------------------- experts
def build(t, h, f, e, k, seed, residual=True, distinct=True):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(e, generator=g)[:k] if distinct else torch.randint(e, (k,), generator=g)
                       for _ in range(t)]).int() if t else torch.empty((0, k), dtype=torch.int32)
    weights = torch.rand(t, k, generator=g)
    return dict(x=values(g, t, h), ids=ids, weights=weights, up=values(g, e, 2 * f, h, std=h ** -0.5),
                down=values(g, e, h, f, std=f ** -0.5), residual=values(g, t, h) if residual else None)


def packed(lib, w):
    return lib.pack_weights(gpu(w).flatten(0, 1)).view(w.shape)


def call(lib, s, act="silu", out=None, up=None, down=None):
    x, res = gpu(s["x"]), gpu(s["residual"])
    out = torch.full_like(x, float("nan")) if out is None else out
    lib.moe_experts(x, gpu(s["ids"]), gpu(s["weights"]), packed(lib, s["up"]) if up is None else up,
                    packed(lib, s["down"]) if down is None else down, out, residual=res, activation=act)
    torch.cuda.synchronize()
    return out


def reference(s, act):
    """The fp64 value, and the bound of an output's error.  Each pair's h = act(g) u carries the fp32
    errors of g and u and one rounding to bf16; these roundings, of F independent values, are at most a
    half step each and uniform, so their weighted sum stays within 6 of its standard deviations (half step
    / sqrt 3 each; 2e-9 of all values lie outside).  Then fp32 sums over F and top_k, and the output's own
    rounding."""
    x, up, down, w = f64(s["x"]), f64(s["up"]), f64(s["down"]), s["weights"].double().numpy()
    ids = s["ids"].numpy()
    e_count, h_size, f = down.shape
    hidden = {}
    ref = ffn.moe_experts(x, ids, w, up, down, None if s["residual"] is None else f64(s["residual"]), act, hidden)
    bound = np.zeros(ref.shape)
    var = np.zeros(ref.shape)
    size = np.abs(f64(s["residual"])) if s["residual"] is not None else np.zeros(ref.shape)
    for (t, j), h in hidden.items():
        e = int(ids[t, j])
        err = sum_error(x[t:t + 1], up[e])[0]
        g, u = up[e, :f] @ x[t], up[e, f:] @ x[t]
        a = ffn.activate(g, act)
        ea = activation_error(g, a, err[:f]) if act != "none" else err[:f]
        eh = np.abs(a) * err[f:] + np.abs(u) * ea + ea * err[f:] + 2 * F32 * np.abs(h)
        d = np.abs(down[e])
        bound[t] += abs(w[t, j]) * (d @ eh + 2 * F32 * chain(f) * (d @ np.abs(h)))
        # pairs of one token with the same expert have the same h, rounded the same way: their weights add up
        # before they are squared (at the first of them)
        same = [i for i in range(ids.shape[1]) if ids[t, i] == e]
        if j == same[0]:
            var[t] += w[t, same].sum() ** 2 * (d ** 2 @ (HALF * (np.abs(h) + eh) / np.sqrt(3.0)) ** 2)
        size[t] += abs(w[t, j]) * (d @ np.abs(h))
    bound += 6 * np.sqrt(var) + 2 * F32 * (ids.shape[1] + 1) * size
    return ref, bound + HALF * (np.abs(ref) + bound) + TINY


def check_experts(lib, s, act="silu", what=""):
    ref, bound = reference(s, act)
    got = call(lib, s, act)
    check(got, ref, bound, f"experts {what}")
    return got


# tokens on both sides of the column tiles, features off the row tiles, one tile of k and odd numbers of them
SHAPES = [(1, 32, 32, 1, 1), (1, 256, 96, 8, 2), (1, 2048, 768, 16, 8), (2, 96, 352, 4, 4), (3, 1024, 160, 60, 4),
          (5, 544, 32, 8, 3), (15, 256, 224, 64, 6), (16, 512, 256, 8, 2), (17, 128, 480, 8, 1), (31, 288, 64, 5, 5),
          (33, 512, 96, 32, 8), (61, 320, 352, 16, 6), (64, 256, 512, 4, 2), (65, 256, 96, 2, 1), (100, 160, 288, 3, 2),
          (129, 256, 64, 16, 4), (200, 512, 128, 8, 2), (256, 128, 96, 1, 1), (256, 64, 32, 200, 16),
          # down products over long ranges, whose waves share row tiles, and few pairs in one kernel
          (20, 64, 2816, 2, 1), (9, 160, 5152, 3, 2), (40, 96, 10272, 3, 2), (8, 96, 5152, 3, 3), (1, 64, 10272, 4, 2),
          (12, 288, 96, 8, 1), (8, 1056, 352, 64, 8), (7, 128, 96, 1024, 9)]


@pytest.mark.parametrize("t,h,f,e,k", SHAPES, ids=["-".join(map(str, s)) for s in SHAPES])
def test_experts(lib, t, h, f, e, k):
    check_experts(lib, build(t, h, f, e, k, seed=sum((t, h, f, e, k))), what=f"{t} tokens")


def reference_on_gpu(s):
    """As reference(), for the larger shapes: fp64 products of the device, an expert at a time, silu; the
    bound without the fp32 errors of h, which are far below its rounding."""
    x, w, ids = s["x"].cuda().double(), s["weights"].cuda().double(), s["ids"].cuda()
    f = s["down"].shape[2]
    ref = torch.zeros_like(x) if s["residual"] is None else s["residual"].cuda().double()
    size, var = ref.abs(), torch.zeros_like(ref)
    for e in range(s["down"].shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        up, down = s["up"][e].cuda().double(), s["down"][e].cuda().double()
        g = x[t] @ up[:f].t()
        h = g / (1 + torch.exp(-g)) * (x[t] @ up[f:].t())
        c = w[t, j][:, None]
        ref.index_add_(0, t, c * (h @ down.t()))
        size.index_add_(0, t, c * (h.abs() @ down.abs().t()))
        var.index_add_(0, t, c ** 2 * ((HALF * h / 3 ** 0.5) ** 2 @ (down ** 2).t()))
    bound = 6 * var.sqrt() + 2 * F32 * (chain(f) + s["ids"].shape[1] + 8) * size
    return f64(ref), f64(bound + HALF * (ref.abs() + bound)) + TINY


# the down products' range cut into 2, 4 and 8 parts; many tokens of one expert
@pytest.mark.parametrize("t,h,f,e,k", [(100, 4096, 2816, 8, 2), (120, 4096, 5152, 8, 2), (90, 16384, 10272, 1, 1),
                                       (256, 2048, 1024, 4, 3)])
def test_experts_of_long_ranges(lib, t, h, f, e, k):
    s = build(t, h, f, e, k, seed=t)
    check(call(lib, s), *reference_on_gpu(s), f"{t} tokens")


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("t", [2, 70])
def test_activations_without_residual(lib, act, t):
    check_experts(lib, build(t, 128, 96, 8, 2, seed=t, residual=False), act, what=act)


@pytest.mark.parametrize("t,e,k", [(1, 3, 3), (3, 1, 16), (4, 2, 16), (16, 2, 4), (40, 3, 8), (64, 1, 1), (21, 2, 3), (90, 2, 2), (256, 1, 16)])
def test_the_same_expert_twice_counts_twice(lib, t, e, k):
    check_experts(lib, build(t, 128, 64, e, k, seed=t + k, distinct=False), what="repeated")


@pytest.mark.parametrize("t", [1, 6, 40, 150])
def test_ids_outside_add_nothing(lib, t):
    s = build(t, 128, 96, 8, 3, seed=t)
    s["ids"][0, 1], s["ids"][t // 2, 0], s["ids"][t - 1] = -1, 8, torch.tensor([2 ** 31 - 1, -2 ** 31, 1 << 20])
    s["weights"][s["ids"] < 0] = float("nan")  # nor do their weights
    s["weights"][s["ids"] >= 8] = float("inf")
    ref, bound = reference({**s, "weights": torch.nan_to_num(s["weights"], 0.0, 0.0, 0.0)}, "silu")
    check(call(lib, s), ref, bound, "ids outside")
    s["ids"][:] = -1
    assert torch.equal(call(lib, s).cpu(), s["residual"])
    s["residual"] = None
    assert (call(lib, s) == 0).all()


@pytest.mark.parametrize("t", [4, 8, 16, 30, 48, 64, 80, 96, 112, 128, 129, 250])
def test_every_token_on_one_expert(lib, t):
    # each number of column tiles, and a second segment
    s = build(t, 256, 160, 16, 2, seed=t)
    s["ids"][:, 0], s["ids"][:, 1] = 11, torch.arange(t) % 3
    check_experts(lib, s, what="one expert")


@pytest.mark.parametrize("t", [5, 50, 200])
def test_in_place_gives_the_same_bits(lib, t):
    s = build(t, 256, 96, 8, 2, seed=t)
    up, down = packed(lib, s["up"]), packed(lib, s["down"])
    want = call(lib, s, up=up, down=down)
    ids, w = gpu(s["ids"]), gpu(s["weights"])
    x, res = gpu(s["x"]), gpu(s["residual"])
    assert torch.equal(lib.moe_experts(x, ids, w, up, down, res, residual=res), want)
    x, res = gpu(s["x"]), gpu(s["residual"])
    assert torch.equal(lib.moe_experts(x, ids, w, up, down, x, residual=res), want)


@pytest.mark.parametrize("t", [6, 45, 150])
def test_what_is_not_finite_stays_with_its_token(lib, t):
    s = build(t, 128, 96, 4, 2, seed=t)
    up, down = packed(lib, s["up"]), packed(lib, s["down"])
    want = call(lib, s, up=up, down=down)
    s["x"][1, 5], s["x"][t - 1, 0] = float("nan"), float("inf")
    got = call(lib, s, up=up, down=down)
    rows = [i for i in range(t) if i not in (1, t - 1)]
    assert torch.equal(got[rows], want[rows]) and not torch.isfinite(got[[1, t - 1]]).any()


@pytest.mark.parametrize("t", [6, 45, 150])
def test_weights_of_experts_that_are_not_asked_for_do_not_matter(lib, t):
    s = build(t, 128, 96, 8, 2, seed=t)
    s["ids"] %= 7
    want = call(lib, s)
    s["up"][7], s["down"][7] = float("nan"), float("inf")
    assert torch.equal(call(lib, s), want)


@pytest.mark.parametrize("t", [6, 16, 45, 150])
def test_weights_that_are_not_finite_reach_the_tokens_that_chose_them(lib, t):
    s = build(t, 128, 96, 8, 2, seed=t)
    s["ids"][s["ids"] == 5] = 6
    s["ids"][1, 0], s["ids"][t - 1, 1] = 5, 5
    want = call(lib, s)
    s["down"][5] = float("nan")
    s["up"][5, 7] = float("inf")
    got = call(lib, s)
    rows = [i for i in range(t) if i not in (1, t - 1)]
    assert torch.equal(got[rows], want[rows]) and torch.isnan(got[[1, t - 1]]).all()


@pytest.mark.parametrize("t,k", [(3, 2), (40, 4), (130, 8)])
def test_graph_replay_with_other_choices(lib, t, k):
    s = build(t, 256, 96, 16, k, seed=t)
    up, down = packed(lib, s["up"]), packed(lib, s["down"])
    x, res, ids, w = gpu(s["x"]), gpu(s["residual"]), gpu(s["ids"]), gpu(s["weights"])
    out = torch.empty_like(x)
    stream = torch.cuda.Stream()
    lib.moe_workspace_reserve(lib.moe_dims(t, 256, 96, 16, k), stream=stream)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        lib.moe_experts(x, ids, w, up, down, out, residual=res)
    for step in range(4):
        other = build(t, 256, 96, 16, k, seed=100 + step)
        ids.copy_(other["ids"] if step % 2 else torch.full_like(other["ids"], step))
        w.copy_(other["weights"])
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, lib.moe_experts(x, ids, w, up, down, torch.empty_like(x), residual=res))
    check(got, *reference({**s, "ids": ids.cpu(), "weights": w.cpu()}, "silu"), "after replays")


def test_two_streams_at_once(lib):
    a, b = build(33, 256, 96, 8, 2, seed=1), build(20, 256, 96, 8, 2, seed=2)
    sets = []
    for s in (a, b):
        sets.append([gpu(s["x"]), gpu(s["ids"]), gpu(s["weights"]), packed(lib, s["up"]), packed(lib, s["down"]), call(lib, s),
                     gpu(s["residual"])])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[torch.empty_like(s[0]) for _ in range(20)] for s in sets]
    torch.cuda.synchronize()
    for i in range(20):
        for s, st, o in zip(sets, streams, outs):
            lib.moe_experts(*s[:5], o[i], residual=s[6], stream=st)
    torch.cuda.synchronize()
    for s, o in zip(sets, outs):
        assert all(torch.equal(t, s[5]) for t in o)


def test_weights_past_4_gib(lib):
    # 110 experts of 2 x 6144 x 2048 elements: 5.5 GB of gate and up weights
    t, h, f, e, k = 4, 2048, 6144, 110, 2
    g = torch.Generator(device="cuda").manual_seed(4)
    up = torch.empty((e, 2 * f, h), dtype=torch.bfloat16, device="cuda").normal_(0, h ** -0.5, generator=g)
    down = torch.empty((e, h, f), dtype=torch.bfloat16, device="cuda").normal_(0, f ** -0.5, generator=g)
    x = torch.empty((t, h), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    pick = [0, 1, e - 1, e - 2]
    ids = torch.tensor([[0, 109], [108, 1], [109, 108], [1, 0]], dtype=torch.int32)
    w = torch.rand(t, k)
    out = lib.moe_experts(x, gpu(ids), gpu(w), lib.pack_weights(up.flatten(0, 1)).view(up.shape),
                          lib.pack_weights(down.flatten(0, 1)).view(down.shape), torch.empty_like(x))
    torch.cuda.synchronize()
    small = dict(x=x, ids=torch.tensor([[pick.index(int(v)) for v in r] for r in ids], dtype=torch.int32), weights=w, up=up[pick],
                 down=down[pick], residual=None)
    check(out, *reference(small, "silu"), "past 4 GiB")


def test_nothing_else_is_written(lib):
    s = build(21, 96, 64, 4, 2, seed=3)
    n = 21 * 96
    buf = torch.full((n + 512,), 7.0, dtype=torch.bfloat16, device="cuda")
    call(lib, s, out=buf[256:256 + n].view(21, 96))
    assert (buf[:256] == 7).all() and (buf[256 + n:] == 7).all()


@pytest.mark.parametrize("t", [6, 40])
def test_offset_rows_give_the_same_bits(lib, t):
    # residual and out need only be 2-byte aligned, ids and weights 4-byte aligned
    s = build(t, 96, 64, 4, 2, seed=t)
    up, down = packed(lib, s["up"]), packed(lib, s["down"])
    want = call(lib, s, up=up, down=down)
    n = t * 96
    buf = torch.empty(2 * n + 8, dtype=torch.bfloat16, device="cuda")
    res, out = buf[1:1 + n].copy_(gpu(s["residual"]).flatten()).view(t, 96), buf[n + 3:2 * n + 3].view(t, 96)
    ids = torch.empty(2 * t + 1, dtype=torch.int32, device="cuda")[1:].view(t, 2).copy_(s["ids"])
    w = torch.empty(2 * t + 3, device="cuda")[3:].view(t, 2).copy_(s["weights"])
    assert torch.equal(lib.moe_experts(gpu(s["x"]), ids, w, up, down, out, residual=res), want)


def test_one_reserve_covers_every_call_below(gpu_lib):
    # captured calls of other sizes fit the workspace that the largest one reserved
    lib, t, h, f, e, k = gpu_lib, 64, 128, 2816, 4, 2
    s = build(t, h, f, e, k, seed=5)
    up, down = packed(lib, s["up"]), packed(lib, s["down"])
    stream = torch.cuda.Stream()
    lib.moe_workspace_reserve(lib.moe_dims(t, h, f, e, k), stream=stream)
    for n, j in ((1, 1), (3, 2), (9, 2), (17, 1), (33, 2), (63, 2), (64, 2)):
        x, ids, w = gpu(s["x"])[:n], gpu(s["ids"])[:n, :j].contiguous(), gpu(s["weights"])[:n, :j].contiguous()
        want = lib.moe_experts(x, ids, w, up, down, torch.empty_like(x))
        out = torch.empty_like(x)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            lib.moe_experts(x, ids, w, up, down, out)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_no_tokens(lib):
    assert call(lib, build(0, 64, 32, 2, 1, seed=0)).shape == (0, 64)
