"""pda_block_norm over as many rows as it takes, where rows times a row's threads pass the 2^32 of one launch:
the same bits as the rows by themselves."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()  # up to 140 GB


def bf(*shape, mean=0.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(mean, generator=g)


def repeated(block, rows):
    """[rows, H]: the block's rows over and over."""
    out = torch.empty((rows, block.shape[1]), dtype=block.dtype, device="cuda")
    for at in range(0, rows, block.shape[0]):
        n = min(block.shape[0], rows - at)
        out[at:at + n] = block[:n]
    return out


def check(got, want):
    for at in range(0, got.shape[0], want.shape[0]):
        n = min(want.shape[0], got.shape[0] - at)
        assert torch.equal(got[at:at + n], want[:n]), f"rows {at} on"


# 1024, 512 and 256 threads a row at their first size past one launch, and rows that end in the middle of a further one
@pytest.mark.parametrize("r,h", [(4194304, 4104), (8388608, 2056), (16777216, 1032), (5000011, 4104)])
def test_more_rows_than_a_launch_has_threads(gpu_lib, r, h):
    block = 65521  # a prime: launches begin at other rows of it
    y, w = bf(block, h, seed=1), bf(h, mean=1.0, seed=2)
    want, _ = gpu_lib.block_norm(y, None, torch.empty_like(y), post_w=w, scale=0.5)
    big = repeated(y, r)
    gpu_lib.block_norm(big, None, big, post_w=w, scale=0.5)
    torch.cuda.synchronize()
    check(big, want)


@pytest.mark.parametrize("gate_rows", [True, False])
def test_every_array_goes_on_with_the_rows(gpu_lib, gate_rows):
    r, h, block = 4194307, 4104, 65521
    y, res, gate = bf(block, h, seed=3), bf(block, h, seed=4), bf(block, h, seed=5)
    gate = gate if gate_rows else gate[0].clone()
    post, pre = bf(h, mean=1.0, seed=6), bf(h, mean=1.0, seed=7)
    kw = dict(post_w=post, pre_w=pre)
    z, n = gpu_lib.block_norm(y, res, torch.empty_like(y), torch.empty_like(y), gate=gate, **kw)
    big, big_res = repeated(y, r), repeated(res, r)
    gpu_lib.block_norm(big, big_res, big_res, big, gate=repeated(gate, r) if gate_rows else gate, **kw)
    torch.cuda.synchronize()
    check(big_res, z)
    check(big, n)
