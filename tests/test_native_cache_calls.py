"""The native marshalling of the cache operators' calls: what it declines goes to the Python checks, and
what it accepts gives what those give."""
import numpy as np
import pytest
import torch

from paper_2606_07665_amd import binding as pda
from test_native_marshalling import _outcome, _Recording, _variants


def _calls(b=3, dev="cpu"):
    """(name, args, kwargs) with accepted arguments."""
    hq, hkv, d, p, m, t = 4, 2, 64, 16, 4, 2
    n = 4 * b
    g = torch.Generator().manual_seed(b)

    def bf(*s):
        return torch.randn(*s, generator=g).to(torch.bfloat16).to(dev)

    def u8(*s):
        return torch.randint(100, 150, s, generator=g, dtype=torch.uint8).to(dev)

    def ints(*s):
        return torch.zeros(s, dtype=torch.int32, device=dev)

    lens = torch.full((b,), 21, dtype=torch.int32, device=dev)
    bt = torch.arange(b * m, dtype=torch.int32).view(b, m).to(dev)
    cache = [u8(n, hkv, 2, p, 16), u8(n, hkv, 2, p), u8(n, hkv, 2, p, 16), u8(n, hkv, 2, p), bt, lens]
    count = torch.ones(n, dtype=torch.int32, device=dev)
    rows = 2 * b
    parents = (torch.arange(rows, dtype=torch.int32) % b).to(dev)
    src, dst = torch.arange(3, dtype=torch.int32).to(dev), torch.arange(3, 6, dtype=torch.int32).to(dev)
    return [
        ("paged_decode_attention_sink", [bf(b, t, hq, d), bf(n, p, hkv, d), bf(n, p, hkv, d), bt, lens, bf(b, t, hq, d), 0.125],
         dict(window=7, sinks=3)),
        ("paged_decode_attention_kv4", [bf(b, t, hq, d), *cache, bf(b, t, hq, d), 0.125], dict(window=7, sinks=3)),
        ("kv4_append", [bf(b, t, hkv, d), bf(b, t, hkv, d), *cache], {}),
        ("kv4_read", [bf(b, t, hkv, d), bf(b, t, hkv, d), *cache], {}),
        ("pages_update", [bt, lens, parents, lens.repeat(2) + 1, count, ints(rows, m), ints(n), ints(rows), ints(rows), ints(2)],
         dict(page_size=p, window=5, sinks=1, num_queries=1)),
        ("pages_compact", [bt, lens, count, ints(b, m), ints(n), ints(n), ints(n), ints(n), ints(2)], dict(page_size=p)),
        ("pages_copy", [[bf(n, p, d), u8(n, 32)], src, dst], dict(count=torch.full((1,), 2, dtype=torch.int32, device=dev))),
    ]


NAMES = [c[0] for c in _calls()]
each = pytest.mark.parametrize("i", range(len(NAMES)), ids=NAMES)


def _results(args):
    return [x.cpu().contiguous().view(torch.uint8).numpy() for a in args for x in (a if isinstance(a, list) else [a])
            if isinstance(x, torch.Tensor)]


@each
def test_cpu_tensors_are_declined_and_refused(i):
    name, args, kwargs = _calls()[i]
    with pytest.raises(ValueError):
        getattr(pda, name)(*args, **kwargs)


def test_wrong_counts_and_kinds_are_declined():
    nat = pda._import_native()
    for f in (nat.attention_sink, nat.attention_kv4, nat.kv4_tokens, nat.pages_update, nat.pages_compact, nat.pages_copy):
        for n in (0, 1, 5, 10, 11, 12, 15, 16):
            assert f(*([None] * n)) == pda._DECLINED
            assert f(*([object()] * n)) == pda._DECLINED
            assert f(*([[]] * n)) == pda._DECLINED
            assert f(*([torch.empty(2, 2, dtype=torch.int32, device="meta")] * n)) == pda._DECLINED


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
