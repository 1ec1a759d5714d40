"""Each form of the experts' kernels at each number of column tiles, their k ranges and rows off a step, a
workgroup and a chunk, against fp64 products of the device.  The plans are pinned, here and for other files'
sizes, so that a change of their rules cannot leave a form untested."""
import pytest
import torch

from _ffn import check
from paper_2606_07665_amd import binding as B
from test_gpu_linear import SHARED
from test_gpu_moe import SHAPES, call, reference_on_gpu

CUS = 256


def plan(t, h, f, e, k):
    p = B.moe_plan(B.moe_dims(t, h, f, e, k), CUS)
    return "joined" if p.joined else ("shared" if p.shared_down else "own") + ("" if p.k_splits == 1 else str(p.k_splits)), \
        "shared" if p.shared_up else "own"


# what test_gpu_moe.py runs: (down, up) of its shapes in order
def test_forms_of_the_shapes():
    joined = {s for s in SHAPES if s[0] <= 8 and s[0] * s[4] <= 64}
    assert [plan(*s) for s in SHAPES] == [("joined" if s in joined else "shared", "own" if s == (40, 96, 10272, 3, 2) else "shared")
                                          for s in SHAPES]
    assert [plan(*s) for s in ((100, 4096, 2816, 8, 2), (120, 4096, 5152, 8, 2), (90, 16384, 10272, 1, 1), (256, 2048, 1024, 4, 3))] == \
        [("own2", "own"), ("own4", "own"), ("own8", "own"), ("own", "own")]


def build(t, h, f, e, k, seed):
    """Every token asks for expert 0, so that its column tiles are known, and for others further on."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def bf(*shape, std=1.0):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0, std, generator=g)
    ids = torch.arange(t, dtype=torch.int32)[:, None] % max(e - 1, 1) + torch.arange(k, dtype=torch.int32)
    ids[:, 0] = 0
    return dict(x=bf(t, h), ids=ids, weights=torch.rand(t, k, generator=g, device="cuda").cpu(), up=bf(e, 2 * f, h, std=h ** -0.5),
                down=bf(e, h, f, std=f ** -0.5), residual=bf(t, h))


PARTS = [(16, 24608, 2592, 4, 2, 2), (49, 24608, 2592, 2, 1, 2), (128, 24608, 2592, 2, 2, 2), (100, 16416, 5184, 1, 1, 4),
         (250, 8224, 5184, 2, 1, 4), (113, 16416, 10336, 1, 1, 8)]
# one to eight column tiles of a segment and a second segment, pairs of few and of many
TOKENS = (6, 9, 16, 17, 31, 33, 48, 49, 64, 65, 80, 81, 96, 97, 112, 113, 128, 129, 145, 250)


def run(t, h, f, e, k, down=None, up=None):
    got = plan(t, h, f, e, k)
    assert (down or got[0], up or got[1]) == got
    s = build(t, h, f, e, k, seed=t + h)
    check(call(B, s), *reference_on_gpu(s), f"{t} tokens")


@pytest.mark.gpu
@pytest.mark.parametrize("t", TOKENS)
@pytest.mark.parametrize("h", [96, 1056])
def test_gate_and_up_of_a_wave_each(gpu_lib, t, h):
    run(t, h, 10272, 4, 2, up="own")


@pytest.mark.gpu
@pytest.mark.parametrize("t", TOKENS[1:])
@pytest.mark.parametrize("f", [96, 1056])
def test_down_of_a_wave_each(gpu_lib, t, f):
    run(t, 20544, f, 4, 2, down="own")


@pytest.mark.gpu
@pytest.mark.parametrize("t,h,f,e,k,parts", PARTS, ids=["-".join(map(str, p[:5])) for p in PARTS])
def test_down_in_parts(gpu_lib, t, h, f, e, k, parts):
    run(t, h, f, e, k, down=f"own{parts}")


@pytest.mark.gpu
@pytest.mark.parametrize("t", TOKENS)
def test_row_tiles_shared(gpu_lib, t):
    run(t, 160, 288, 4, 2, "joined" if t <= 8 else "shared", "shared")


# the parts of k of test_gpu_linear.py's gated products that share their activations
def test_parts_of_the_gated_products():
    parts = [B.linear_plan(B.linear_dims(b, k, n // 32 * 16, "silu", True), CUS).k_splits for b, k, n, _ in SHARED]
    assert parts == [1, 1, 1, 1, 5, 3, 1, 1, 1, 1, 2, 4, 5, 6, 1, 6, 1, 1, 1]
