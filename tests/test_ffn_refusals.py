"""Argument checks of the feed-forward operators' entry points (before any HIP call, so no GPU), the
planner of linear products, and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_2606_07665_amd import binding as B

NULL, SHAPE, UNSUPPORTED, SCALE, ALIGN, LAYOUT = 1, 2, 3, 4, 5, 8
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return B.load()


def refused(rc, code, text):
    assert rc == code and text in B.last_error(), (rc, B.last_error())


def linear(lib, x=MB, w=2 * MB, bias=0, residual=0, out=64 * MB, **dims):
    d = B.LinearDims(**dict(dict(batch=4, in_features=64, out_features=32, activation=0, gated=0, out_f32=0), **dims))
    return lib.pda_linear(x, w, bias, residual, out, ctypes.byref(d), None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(batch=-1), SHAPE, "batch"), (dict(batch=257), UNSUPPORTED, "batch"),
    (dict(in_features=0), SHAPE, "positive"), (dict(out_features=-16), SHAPE, "positive"),
    (dict(in_features=48), UNSUPPORTED, "in_features"), (dict(in_features=65568), UNSUPPORTED, "in_features"),
    (dict(out_features=24), UNSUPPORTED, "out_features"), (dict(out_features=262160), UNSUPPORTED, "out_features"),
    (dict(activation=5), UNSUPPORTED, "activation"), (dict(activation=-1), UNSUPPORTED, "activation"),
    (dict(gated=2), SHAPE, "gated"), (dict(out_f32=-1), SHAPE, "out_f32"),
    (dict(gated=1, in_features=65536, out_features=16384), UNSUPPORTED, "gated"),
    (dict(x=0), NULL, "NULL"), (dict(w=0), NULL, "NULL"), (dict(out=0), NULL, "NULL"),
    (dict(x=MB + 8), ALIGN, "16-byte"), (dict(w=MB + 2), ALIGN, "16-byte"), (dict(bias=33), ALIGN, "2-byte"),
    (dict(residual=33), ALIGN, "2-byte"), (dict(out=64 * MB + 2, out_f32=1), ALIGN, "4-byte"),
    (dict(out=MB), LAYOUT, "x"), (dict(out=MB + 511), ALIGN, "2-byte"), (dict(out=MB - 2), LAYOUT, "x"),
    (dict(out=2 * MB + 4094), LAYOUT, "w_packed"), (dict(bias=64 * MB, out=64 * MB), LAYOUT, "bias"),
    (dict(residual=64 * MB + 2), LAYOUT, "residual"), (dict(residual=64 * MB, out_f32=1), LAYOUT, "residual"),
])
def test_linear(lib, kw, code, text):
    refused(linear(lib, **kw), code, text)


def test_null_dims(lib):
    refused(lib.pda_linear(16, 16, 0, 0, 16, None, None), NULL, "dims")
    refused(lib.pda_moe_route(16, 0, 16, 16, None, None), NULL, "dims")
    refused(lib.pda_moe_experts(*[16] * 7, None, None), NULL, "dims")
    refused(lib.pda_block_norm(*[16] * 7, None, None), NULL, "dims")
    for fn in (lib.pda_linear_workspace_reserve, lib.pda_moe_workspace_reserve):
        refused(fn(None, None), NULL, "dims")
    refused(lib.pda_linear_plan(None, 256, ctypes.byref(B.Projection())), NULL, "dims")
    refused(lib.pda_linear_plan(ctypes.byref(B.linear_dims(1, 32, 16)), 256, None), NULL, "output")
    refused(lib.pda_linear_plan(ctypes.byref(B.linear_dims(1, 32, 16)), 0, ctypes.byref(B.Projection())), SHAPE, "num_cus")


def route(lib, logits=MB, bias=0, ids=2 * MB, weights=3 * MB, **dims):
    d = B.RouteDims(**dict(dict(tokens=4, num_experts=16, top_k=2, logit_stride=16, sigmoid=0, renormalise=1, scale=1.0), **dims))
    return lib.pda_moe_route(logits, bias, ids, weights, ctypes.byref(d), None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(tokens=-1), SHAPE, "tokens"), (dict(tokens=(1 << 20) + 1), UNSUPPORTED, "tokens"),
    (dict(num_experts=0), SHAPE, "positive"), (dict(top_k=0), SHAPE, "positive"),
    (dict(num_experts=1025, logit_stride=1025), UNSUPPORTED, "num_experts"), (dict(top_k=17), UNSUPPORTED, "top_k"),
    (dict(num_experts=4, top_k=5), SHAPE, "top_k"), (dict(logit_stride=15), LAYOUT, "logit_stride"),
    (dict(sigmoid=2), SHAPE, "sigmoid"), (dict(renormalise=-1), SHAPE, "renormalise"),
    (dict(scale=float("inf")), SCALE, "scale"), (dict(scale=float("nan")), SCALE, "scale"),
    (dict(logits=0), NULL, "NULL"), (dict(ids=0), NULL, "NULL"), (dict(weights=0), NULL, "NULL"),
    (dict(logits=MB + 2), ALIGN, "4-byte"), (dict(bias=6), ALIGN, "4-byte"), (dict(ids=2 * MB + 1), ALIGN, "4-byte"),
    (dict(ids=MB + 252), LAYOUT, "logits"), (dict(weights=2 * MB + 28), LAYOUT, "expert_weights"),
    (dict(weights=MB + 60), LAYOUT, "logits"), (dict(bias=3 * MB), LAYOUT, "select_bias"),
])
def test_route(lib, kw, code, text):
    refused(route(lib, **kw), code, text)


def experts(lib, x=MB, ids=2 * MB, weights=3 * MB, up=4 * MB, down=8 * MB, residual=0, out=64 * MB, **dims):
    d = B.MoeDims(**dict(dict(tokens=4, hidden=64, inter=32, num_experts=8, top_k=2, activation=1), **dims))
    return lib.pda_moe_experts(x, ids, weights, up, down, residual, out, ctypes.byref(d), None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(tokens=-1), SHAPE, "tokens"), (dict(tokens=257), UNSUPPORTED, "tokens"),
    (dict(hidden=0), SHAPE, "positive"), (dict(inter=-32), SHAPE, "positive"), (dict(num_experts=0), SHAPE, "positive"),
    (dict(top_k=0), SHAPE, "positive"), (dict(hidden=48), UNSUPPORTED, "hidden"), (dict(hidden=32800), UNSUPPORTED, "hidden"),
    (dict(inter=16), UNSUPPORTED, "inter"), (dict(inter=65568), UNSUPPORTED, "inter"),
    (dict(num_experts=1025), UNSUPPORTED, "num_experts"), (dict(top_k=17), UNSUPPORTED, "top_k"),
    (dict(activation=5), UNSUPPORTED, "activation"),
    (dict(x=0), NULL, "NULL"), (dict(ids=0), NULL, "NULL"), (dict(weights=0), NULL, "NULL"), (dict(up=0), NULL, "NULL"),
    (dict(down=0), NULL, "NULL"), (dict(out=0), NULL, "NULL"),
    (dict(x=MB + 8), ALIGN, "16-byte"), (dict(up=4 * MB + 8), ALIGN, "16-byte"), (dict(down=8 * MB + 8), ALIGN, "16-byte"),
    (dict(ids=2 * MB + 2), ALIGN, "4-byte"), (dict(weights=3 * MB + 2), ALIGN, "4-byte"), (dict(out=64 * MB + 1), ALIGN, "2-byte"),
    (dict(out=MB + 2), LAYOUT, "x"), (dict(residual=64 * MB - 2), LAYOUT, "residual"), (dict(out=2 * MB), LAYOUT, "expert_ids"),
    (dict(out=3 * MB), LAYOUT, "expert_weights"), (dict(out=4 * MB), LAYOUT, "w_gate_up"), (dict(out=8 * MB), LAYOUT, "w_down"),
])
def test_experts(lib, kw, code, text):
    refused(experts(lib, **kw), code, text)


def norm(lib, y=MB, residual=0, post=0, pre=3 * MB, gate=0, z=4 * MB, h=5 * MB, **dims):
    d = B.BlockNormDims(**dict(dict(rows=4, hidden=64, gate_rows=0, scale=1.0, weight_offset=0.0, eps=1e-5), **dims))
    return lib.pda_block_norm(y, residual, post, pre, gate, z, h, ctypes.byref(d), None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(rows=-1), SHAPE, "rows"), (dict(rows=(1 << 24) + 1), UNSUPPORTED, "rows"), (dict(hidden=0), SHAPE, "hidden"),
    (dict(hidden=12), UNSUPPORTED, "hidden"), (dict(hidden=32776), UNSUPPORTED, "hidden"),
    (dict(gate_rows=2), SHAPE, "gate_rows"), (dict(scale=float("nan")), SCALE, "finite"),
    (dict(weight_offset=float("inf")), SCALE, "finite"), (dict(eps=-1e-6), SCALE, "eps"), (dict(eps=float("inf")), SCALE, "eps"),
    (dict(pre=0), NULL, "pre_w"), (dict(h=0), NULL, "normed_out"), (dict(y=0), NULL, "NULL"), (dict(z=0), NULL, "NULL"),
    (dict(post=33), ALIGN, "2-byte"), (dict(h=5 * MB + 1), ALIGN, "2-byte"),
    (dict(z=MB + 16), LAYOUT, "y"), (dict(residual=4 * MB + 2), LAYOUT, "residual"), (dict(z=3 * MB), LAYOUT, "pre_w"),
    (dict(post=5 * MB), LAYOUT, "post_w"), (dict(gate=4 * MB), LAYOUT, "gate"),
    (dict(gate=4 * MB - 256, gate_rows=1), LAYOUT, "gate"), (dict(h=4 * MB + 510), LAYOUT, "normed_out overlaps residual_out"),
    (dict(z=MB, h=MB), LAYOUT, "normed_out overlaps residual_out"),
])
def test_block_norm(lib, kw, code, text):
    refused(norm(lib, **kw), code, text)


def test_empty_calls_are_no_ops(lib):
    assert linear(lib, x=0, w=0, out=0, batch=0) == 0
    assert route(lib, logits=0, ids=0, weights=0, tokens=0) == 0
    assert experts(lib, x=0, ids=0, weights=0, up=0, down=0, out=0, tokens=0) == 0
    assert norm(lib, y=0, z=0, pre=0, rows=0) == 0
    assert lib.pda_linear_workspace_reserve(ctypes.byref(B.linear_dims(0, 32, 16)), None) == 0
    assert lib.pda_moe_workspace_reserve(ctypes.byref(B.moe_dims(0, 32, 32, 1, 1)), None) == 0
    assert B.linear_plan(B.linear_dims(0, 32, 16)).workgroups == 0


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("k,n", [(32, 16), (4096, 128), (4096, 14336), (8192, 1040), (512, 262144)])
def test_linear_plans(gated, k, n):
    bytes_before = 0
    for b in (1, 7, 16, 17, 33, 64, 65, 130, 200, 256):
        p = B.linear_plan(B.linear_dims(b, k, n, "silu", gated))
        rows = 2 * n if gated else n
        assert p.row_tiles * 16 * (p.workgroups // (p.col_groups * p.k_splits)) >= rows
        assert p.col_tiles * 16 * p.col_groups >= b
        # a split product ends in a kernel of its own, and so does a gated one without pairs of row tiles
        assert p.fused == (p.k_splits == 1 and (not gated or p.row_tiles % 2 == 0))
        assert p.fused or p.workspace_bytes >= 4 * p.k_splits * b * rows
        assert p.workspace_bytes >= bytes_before  # one reserve covers every smaller batch
        bytes_before = p.workspace_bytes


# ---- the binding's checks: CPU tensors reach them
def bf(*s):
    return torch.zeros(s, dtype=torch.bfloat16)


def calls():
    i32, f32 = torch.int32, torch.float32
    return dict(
        linear=(B.linear, dict(x=bf(4, 64), w_packed=bf(32, 64), out=bf(4, 32), bias=bf(32), residual=bf(4, 32))),
        moe_route=(B.moe_route, dict(logits=torch.zeros(4, 16), expert_ids=torch.zeros(4, 2, dtype=i32),
                                     expert_weights=torch.zeros(4, 2), select_bias=torch.zeros(16))),
        moe_experts=(B.moe_experts, dict(x=bf(4, 64), expert_ids=torch.zeros(4, 2, dtype=i32), expert_weights=torch.zeros(4, 2),
                                         w_gate_up=bf(3, 64, 64), w_down=bf(3, 64, 32), out=bf(4, 64), residual=bf(4, 64))),
        block_norm=(B.block_norm, dict(y=bf(4, 64), residual=bf(4, 64), residual_out=bf(4, 64), normed_out=bf(4, 64),
                                       post_w=bf(64), pre_w=bf(64), gate=bf(4, 64))))


@pytest.mark.parametrize("name,over,kind,text", [
    ("linear", dict(w_packed=bf(32, 96)), ValueError, "w_packed"), ("linear", dict(w_packed=bf(48, 64)), ValueError, "w_packed"),
    ("linear", dict(gated=True), ValueError, "w_packed"), ("linear", dict(bias=bf(64)), ValueError, "bias"),
    ("linear", dict(residual=bf(3, 32)), ValueError, "residual"), ("linear", dict(out=bf(5, 32)), ValueError, "out"),
    ("linear", dict(out=torch.zeros(4, 32, dtype=torch.float16)), TypeError, "out"),
    ("linear", dict(x=torch.zeros(4, 64)), TypeError, "x"), ("linear", dict(activation="tanh"), ValueError, "activation"),
    ("linear", dict(), ValueError, "GPU"),
    ("moe_route", dict(logits=torch.zeros(5, 16)), ValueError, "expert_ids .* T = 5"),
    ("moe_route", dict(logits=torch.zeros(4, 15)), ValueError, "select_bias .* E = 15"),
    ("moe_route", dict(logits=torch.zeros(16)), ValueError, "logits"),
    ("moe_route", dict(scoring="max"), ValueError, "scoring"),
    ("moe_route", dict(expert_weights=torch.zeros(4, 3)), ValueError, "expert_weights"),
    ("moe_route", dict(expert_ids=torch.zeros(4, 2, dtype=torch.int64)), TypeError, "expert_ids"),
    ("moe_route", dict(), ValueError, "GPU"),
    ("moe_experts", dict(w_gate_up=bf(3, 32, 64)), ValueError, "w_gate_up"),
    ("moe_experts", dict(w_gate_up=bf(2, 64, 64)), ValueError, "w_gate_up"),
    ("moe_experts", dict(w_down=bf(3, 32, 32)), ValueError, "w_down"), ("moe_experts", dict(out=bf(4, 32)), ValueError, "out"),
    ("moe_experts", dict(expert_ids=torch.zeros(4, dtype=torch.int32)), ValueError, "expert_ids"),
    ("moe_experts", dict(activation=None), ValueError, "activation"), ("moe_experts", dict(), ValueError, "GPU"),
    ("block_norm", dict(gate=bf(5, 64)), ValueError, "gate"), ("block_norm", dict(gate=bf(32)), ValueError, "gate"),
    ("block_norm", dict(post_w=bf(32)), ValueError, "post_w"), ("block_norm", dict(pre_w=None), ValueError, "both"),
    ("block_norm", dict(normed_out=None), ValueError, "both"), ("block_norm", dict(residual=bf(4, 32)), ValueError, "residual"),
    ("block_norm", dict(y=torch.zeros(4, 64)), TypeError, "y"), ("block_norm", dict(), ValueError, "GPU"),
])
def test_binding(name, over, kind, text):
    fn, kw = calls()[name]
    with pytest.raises(kind, match=text):
        fn(**dict(kw, **over))


def test_dims_past_32_bits_are_refused():
    for make in (lambda n: B.linear_dims(n, 32, 16), lambda n: B.linear_dims(1, 32, n), lambda n: B.moe_dims(1, 32, n, 1, 1)):
        with pytest.raises(ValueError):
            make(1 << 32)
