"""GPU parity of pda_block_norm against the fp64 oracle."""
import numpy as np
import pytest
import torch

from _ffn import F32, HALF, TINY, check, f64, gpu, values
from oracle import ffn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(gpu_lib):
    return gpu_lib


def build(r, h, post, pre, gate, residual, offset, seed):
    g = torch.Generator().manual_seed(seed + r + h)
    w = lambda on: values(g, h, mean=1.0 - offset, std=0.2) if on else None
    return dict(y=values(g, r, h, std=3.0), residual=values(g, r, h) if residual else None, post_w=w(post), pre_w=w(pre),
                gate=None if gate is None else values(g, h) if gate == "features" else values(g, r, h))


def reference(s, scale, offset, eps):
    a = {k: None if t is None else f64(t) for k, t in s.items()}
    z, h = ffn.block_norm(a["y"], a["residual"], a["post_w"], a["pre_w"], a["gate"], float(np.float32(scale)), offset,
                          float(np.float32(eps)))
    # a mean of squares in fp32 is off by at most the roundings in a row (32 in a thread, 6 and 16 over
    # the workgroup, and a few), its root by half as many steps; then six products and sums
    norm = (64 / 2 + 8) * F32
    part = z - (0.0 if a["residual"] is None else a["residual"])
    ez = norm * np.abs(part) + 4 * F32 * (np.abs(z) + np.abs(part))
    bz = ez + HALF * (np.abs(z) + ez) + TINY
    if h is None:
        return (z, bz), None
    rms = np.sqrt(np.mean(z * z, axis=1, keepdims=True) + float(np.float32(eps)))
    eh = norm * np.abs(h) + (ez + np.abs(z) * np.max(ez / rms, axis=1, keepdims=True)) / rms * np.abs(a["pre_w"] + offset)
    return (z, bz), (h, eh + HALF * (np.abs(h) + eh) + TINY)


def run(lib, s, scale=1.0, offset=0.0, eps=1e-6):
    d = {k: gpu(t) for k, t in s.items()}
    z = torch.full_like(d["y"], float("nan"))
    h = torch.full_like(d["y"], float("nan")) if d["pre_w"] is not None else None
    got = lib.block_norm(d["y"], d["residual"], z, h, post_w=d["post_w"], pre_w=d["pre_w"], gate=d["gate"], scale=scale,
                         weight_offset=offset, eps=eps)
    assert got[0] is z and got[1] is h
    torch.cuda.synchronize()
    return z, h


@pytest.mark.parametrize("post,pre,gate,residual,scale,offset", [
    (False, False, None, False, 1.0, 0.0), (True, True, None, True, 1.0, 0.0), (False, True, "features", True, 0.25, 0.0),
    (True, False, "rows", True, -1.5, 1.0), (True, True, "rows", False, 0.7, 1.0), (False, True, "rows", True, 0.0, 0.0)])
@pytest.mark.parametrize("r,h", [(1, 8), (3, 512), (2, 520), (7, 2048), (5, 2056), (4, 4096), (3, 4104), (2, 8192), (3, 8200),
                                 (2, 16384), (2, 16392), (1, 32768)])
def test_block_norm(lib, r, h, post, pre, gate, residual, scale, offset):
    s = build(r, h, post, pre, gate, residual, offset, seed=1)
    z, hn = run(lib, s, scale, offset)
    ref_z, ref_h = reference(s, scale, offset, 1e-6)
    check(z, *ref_z, f"z {r} x {h}")
    if pre:
        check(hn, *ref_h, f"h {r} x {h}")


def test_many_rows(lib):
    s = build(70000, 64, True, True, "rows", True, 0.0, seed=2)
    z, h = run(lib, s)
    ref_z, ref_h = reference(s, 1.0, 0.0, 1e-6)
    check(z, *ref_z, "z")
    check(h, *ref_h, "h")


def test_rows_past_32_bit_offsets(lib):
    # 131080 x 32768 elements: the last rows lie 8 GiB on
    r, h = 131080, 32768
    y = torch.zeros((r, h), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(h, dtype=torch.bfloat16, device="cuda")
    y[-1] = torch.randn(h, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    want = run(lib, dict(y=y[-1:].clone(), residual=None, post_w=None, pre_w=w, gate=None))
    z = torch.full_like(y, 7.0)
    lib.block_norm(y, None, z, y, pre_w=w, eps=1e-6)
    torch.cuda.synchronize()
    assert torch.equal(z[-1:], want[0]) and torch.equal(y[-1:], want[1])
    assert (z[-2] == 0).all() and (z[r // 2] == 0).all()


@pytest.mark.parametrize("h", [256, 5120, 20480])
def test_outputs_in_the_place_of_inputs(lib, h):
    s = build(6, h, True, True, "features", True, 0.0, seed=3)
    want = run(lib, s)
    d = {k: gpu(t) for k, t in s.items()}
    kw = dict(post_w=d["post_w"], pre_w=d["pre_w"], gate=d["gate"], eps=1e-6)
    for z_in, h_in in (("residual", "y"), ("y", "residual"), ("residual", None), ("y", None)):
        y, r = d["y"].clone(), d["residual"].clone()
        at = dict(y=y, residual=r)
        z, hn = lib.block_norm(y, r, at[z_in], at[h_in] if h_in else torch.empty_like(y), **kw)
        assert torch.equal(z, want[0]) and torch.equal(hn, want[1]), (z_in, h_in)


def test_zero_rows_and_what_is_not_finite(lib):
    s = build(6, 512, True, True, None, True, 0.0, seed=4)
    s["y"][0], s["residual"][0] = 0.0, 0.0
    s["y"][2, 9], s["residual"][4, 3] = float("nan"), float("inf")
    z, h = run(lib, s)
    assert (z[0] == 0).all() and (h[0] == 0).all()
    assert not torch.isfinite(z[2]).any() and torch.isnan(h[4, 3]) and not torch.isfinite(z[4, 3])
    clean = {k: None if t is None else t.clone() for k, t in s.items()}
    clean["y"][2, 9], clean["residual"][4, 3] = 0.0, 0.0
    want = run(lib, clean)
    for i in (0, 1, 3, 5):
        assert torch.equal(z[i], want[0][i]) and torch.equal(h[i], want[1][i])


def test_offset_rows_give_the_same_bits(lib):
    s = build(3, 264, True, True, "rows", True, 0.0, seed=5)
    want = run(lib, s)
    n = 3 * 264
    buf = torch.full((5 * n + 2 * 264 + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    at, d = 1, {}
    for k, t in s.items():
        d[k] = buf[at:at + t.numel()].copy_(t.cuda().flatten()).view(t.shape)
        at += t.numel() + (3 if t.dim() == 1 else 1)
    z, h = buf[at:at + n].view(3, 264), buf[at + n + 1:at + 2 * n + 1].view(3, 264)
    lib.block_norm(d["y"], d["residual"], z, h, post_w=d["post_w"], pre_w=d["pre_w"], gate=d["gate"], eps=1e-6)
    assert torch.equal(z, want[0]) and torch.equal(h, want[1])
    assert buf[at - 1] == 7 and buf[at + n] == 7 and (buf[at + 2 * n + 1:] == 7).all()


def test_graph_replay(lib):
    s = {k: gpu(t) for k, t in build(9, 4096, True, True, None, True, 0.0, seed=6).items()}
    z, h = torch.empty_like(s["y"]), torch.empty_like(s["y"])
    call = lambda: lib.block_norm(s["y"], s["residual"], z, h, post_w=s["post_w"], pre_w=s["pre_w"])
    call()
    want = z.clone(), h.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        z.zero_(), h.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want[0]) and torch.equal(h, want[1])


def test_no_rows(lib):
    s = build(0, 64, True, True, None, True, 0.0, seed=7)
    assert run(lib, s)[0].shape == (0, 64)
