"""The workspace of the experts' products: what a call writes, by its plan, and what it asks for, which
covers every smaller call.  On the GPU a call that fits its stream's workspace is captured with it, and
leaves it to the graphs that were captured before."""
import ctypes
import random

import pytest

from paper_2606_07665_amd import binding as B

CUS = (64, 256, 304)


def up256(n):
    return -(-n // 256) * 256


def written(d, p):
    """h in bf16, and unless the down products end in the kernel that adds them, fp32 sums of each part."""
    pairs = d.tokens * d.top_k
    return up256(2 * pairs * d.inter) + up256(0 if p.joined else 4 * p.k_splits * pairs * d.hidden)


def drawn(rng):
    e = rng.choice((1, 2, 8, 60, 256, 1024))
    return B.moe_dims(rng.randint(1, 256), 32 * rng.choice((1, 3, 64, 128, 300, 1024)), 32 * rng.choice((1, 12, 44, 161, 448, 2048)),
                      e, rng.randint(1, 16))


def test_what_a_call_writes():
    rng = random.Random(1)
    forms = set()
    for _ in range(4000):
        d, cus = drawn(rng), rng.choice(CUS)
        p = B.moe_plan(d, cus)
        forms.add((p.joined, p.shared_up, p.shared_down, p.k_splits))
        assert p.joined == (d.tokens <= 8 and d.tokens * d.top_k <= 64)
        assert p.k_splits in (1, 2, 4, 8) and (p.k_splits == 1 or not (p.joined or p.shared_down))
        assert p.call_bytes == written(d, p) <= p.workspace_bytes
    assert {f[3] for f in forms} == {1, 2, 4, 8} and len({f[:3] for f in forms}) == 6


def test_the_workspace_covers_smaller_calls():
    rng = random.Random(2)
    for _ in range(400):
        d, cus = drawn(rng), rng.choice(CUS)
        most = B.moe_plan(d, cus).workspace_bytes
        for _ in range(12):
            less = B.moe_dims(rng.randint(1, d.tokens), d.hidden, d.inter, d.num_experts, rng.randint(1, d.top_k))
            p = B.moe_plan(less, cus)
            assert p.call_bytes <= p.workspace_bytes <= most


def test_plan_arguments():
    lib, p = B.load(), B.Experts()
    d = B.moe_dims(4, 64, 32, 8, 2)
    for dims, cus, out, code in ((None, 256, p, 1), (d, 256, None, 1), (d, 0, p, 2), (B.moe_dims(-1, 64, 32, 8, 2), 256, p, 2),
                                 (B.moe_dims(4, 48, 32, 8, 2), 256, p, 3), (B.moe_dims(4, 64, 32, 8, 17), 256, p, 3)):
        assert lib.pda_moe_plan(dims and ctypes.byref(dims), cus, out and ctypes.byref(out)) == code
    p = B.moe_plan(B.moe_dims(0, 64, 32, 8, 2))
    assert (p.joined, p.k_splits, p.call_bytes, p.workspace_bytes) == (0, 0, 0, 0)


# (tokens, hidden, inter, experts, top_k): h alone; sums of whole ranges, a wave's row tiles shared or not; of two parts
CALLS = [(1, 8192, 64, 8, 8), (16, 2048, 96, 8, 2), (128, 2048, 256, 64, 4), (100, 4096, 2816, 8, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("t,h,f,e,k", CALLS, ids=["-".join(map(str, c)) for c in CALLS])
def test_a_call_that_fits_leaves_the_workspace_to_earlier_graphs(gpu_lib, t, h, f, e, k):
    """A product split along k is captured on a stream whose workspace holds what the experts' call writes
    but not what it asks for; that call is captured there as well, then made eagerly, and both graphs still
    write to a buffer of their own."""
    import torch
    lib = gpu_lib
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    plan = lib.moe_plan(lib.moe_dims(t, h, f, e, k), cus)
    lk = 8192

    # the first split product whose buffer (a quarter more than it asks for) holds the call's bytes
    def buffer(b, n):
        p = lib.linear_plan(lib.linear_dims(b, lk, n), cus)
        return p.workspace_bytes * 5 // 4 if not p.fused else 0
    b, n = next((b, n) for b in (24, 200) for n in range(640, 16384, 16) if buffer(b, n) >= plan.call_bytes)
    assert plan.call_bytes <= buffer(b, n) < plan.workspace_bytes
    gen = torch.Generator(device="cuda").manual_seed(t)

    def bf(*shape, std=1.0):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0, std, generator=gen)
    lw, lx, lout = lib.pack_weights(bf(n, lk, std=lk ** -0.5)), bf(b, lk), bf(b, n)
    up, down = bf(e, 2 * f, h, std=h ** -0.5), bf(e, h, f, std=f ** -0.5)
    up, down = (lib.pack_weights(w.flatten(0, 1)).view(w.shape) for w in (up, down))
    x, out, w = bf(t, h), bf(t, h), torch.rand(t, k, device="cuda")
    ids = torch.randint(e, (t, k), dtype=torch.int32, device="cuda", generator=gen)

    def linear(stream=None):
        lib.linear(lx, lw, lout, stream=stream)

    def experts(stream=None):
        lib.moe_experts(x, ids, w, up, down, out, stream=stream)
    linear(), experts()
    torch.cuda.synchronize()
    want = lout.clone(), out.clone()
    lib.release_workspaces()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    lib.linear_workspace_reserve(lib.linear_dims(b, lk, n), stream=s)
    graphs = []
    for call in (linear, experts):
        print("capture", call.__name__, flush=True)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call(s)
        graphs.append(g)
    for _ in range(2):
        experts(s)  # grows the stream's workspace for larger calls, and keeps the graphs'
        torch.cuda.synchronize()
        assert torch.equal(out, want[1])
        others = [torch.full((1 << 20,), 7, dtype=torch.int32, device="cuda") for _ in range(32)]
        for g, got, ref in zip(graphs, (lout, out), want):
            got.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, ref)
        assert all(bool((o == 7).all()) for o in others)
        del others
        torch.cuda.empty_cache()
    del graphs, g
    lib.release_workspaces()
