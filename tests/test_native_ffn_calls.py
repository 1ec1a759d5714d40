"""The native marshalling of the feed-forward calls: what it declines goes to the Python checks, and what
it accepts gives what those give."""
import numpy as np
import pytest
import torch

from paper_2606_07665_amd import binding as pda
from test_native_marshalling import _outcome, _Recording, _variants


def _calls(b=3, dev="cpu"):
    """(name, args, kwargs) with accepted arguments."""
    g = torch.Generator().manual_seed(b)

    def bf(*s):
        return torch.randn(*s, generator=g).to(torch.bfloat16).to(dev)

    def f32(*s):
        return torch.randn(*s, generator=g).to(dev)

    ids = (torch.arange(2 * b, dtype=torch.int32) % 3).view(b, 2).to(dev)
    return [
        ("linear", [bf(b, 64), bf(32, 64), bf(b, 32)], dict(bias=bf(32), residual=bf(b, 32), activation="gelu")),
        ("linear", [bf(b, 64), bf(64, 64), f32(b, 32)], dict(bias=bf(64), activation="silu", gated=True)),
        ("moe_route", [f32(b, 20), torch.zeros_like(ids), f32(b, 2)], dict(scoring="sigmoid", renormalise=False,
                                                                          select_bias=f32(20), scale=1.5)),
        ("moe_route", [f32(b, 24)[:, :20], torch.zeros_like(ids), f32(b, 2)], {}),
        ("moe_experts", [bf(b, 64), ids, f32(b, 2), bf(3, 64, 64), bf(3, 64, 32), bf(b, 64)], dict(residual=bf(b, 64))),
        ("block_norm", [bf(b, 64), bf(b, 64), bf(b, 64), bf(b, 64)], dict(post_w=bf(64), pre_w=bf(64), gate=bf(b, 64), scale=0.5,
                                                                          weight_offset=1.0, eps=1e-6)),
        ("block_norm", [bf(b, 64), None, bf(b, 64)], dict(gate=bf(64))),
    ]


NAMES = ["%s%d" % (c[0], i) for i, c in enumerate(_calls())]
each = pytest.mark.parametrize("i", range(len(NAMES)), ids=NAMES)


def _results(args):
    return [a.cpu().contiguous().view(torch.uint8).numpy() for a in args if isinstance(a, torch.Tensor)]


@each
def test_cpu_tensors_are_declined_and_refused(i):
    name, args, kwargs = _calls()[i]
    with pytest.raises(ValueError):
        getattr(pda, name)(*args, **kwargs)


def test_wrong_counts_and_kinds_are_declined():
    nat = pda._import_native()
    for f in (nat.linear, nat.moe_route, nat.moe_experts, nat.block_norm):
        for n in (0, 1, 7, 8, 9, 11, 12):
            assert f(*([None] * n)) == pda._DECLINED
            assert f(*([object()] * n)) == pda._DECLINED
            assert f(*([3] * n)) == pda._DECLINED
            for dt in (torch.bfloat16, torch.float32, torch.int32):
                assert f(*([torch.empty(2, 2, dtype=dt, device="meta")] * n)) == pda._DECLINED


@pytest.mark.gpu
@each
def test_the_plain_call_is_taken_natively(gpu_lib, monkeypatch, i):
    rec = _Recording(pda._import_native())
    monkeypatch.setattr(pda, "_nat", rec)
    name, args, kwargs = _calls(5, "cuda")[i]
    getattr(pda, name)(*args, **kwargs)
    torch.cuda.synchronize()
    assert rec.answers == [pda.PDA_OK]


@pytest.mark.gpu
@each
def test_the_stream_is_that_of_the_checks(gpu_lib, monkeypatch, i):
    name, args, kwargs = _calls(5, "cuda")[i]
    rec = _Recording(pda._import_native(current_device=lambda: 1))
    monkeypatch.setattr(pda, "_nat", rec)
    getattr(pda, name)(*args, **kwargs)
    getattr(pda, name)(*args, stream=torch.cuda.current_stream(), **kwargs)
    torch.cuda.synchronize()
    assert rec.answers == [pda._DECLINED, pda.PDA_OK]


@pytest.mark.gpu
@each
def test_native_and_python_paths_agree(gpu_lib, monkeypatch, i):
    got = {}
    for path in ("native", "python"):
        monkeypatch.setattr(pda, "_nat", pda._import_native() if path == "native" else pda._Declining())
        name, args, kwargs = _calls(5, "cuda")[i]
        getattr(pda, name)(*args, **kwargs)
        torch.cuda.synchronize()
        got[path] = _results(args)
    for a, b in zip(got["native"], got["python"]):
        assert np.array_equal(a, b)
    name, args, kwargs = _calls(5, "cuda")[i]
    for what, (a, k) in _variants(args, kwargs):
        seen = []
        for path in ("native", "python"):
            monkeypatch.setattr(pda, "_nat", pda._import_native() if path == "native" else pda._Declining())
            seen.append(_outcome(name, a, k))
        assert seen[0] == seen[1], f"{name}, {what}: {seen}"
    torch.cuda.synchronize()
