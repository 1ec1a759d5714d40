"""A decode layer's operators run together, as a serving loop runs them: prelude with the append, attention,
output projection, then the feed-forward half (dense, and a mixture of experts) up to the next layer's
normed input -- eagerly, and captured into one graph -- each step against the oracle on what came before it."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from _ffn import F32, check, f64, linear_error, values
from _gpu import bf16_ulps
from oracle import ffn
from test_gpu_block_norm import reference as norm_reference
from test_gpu_moe import reference as experts_reference

pytestmark = pytest.mark.gpu

H, HQ, HKV, D, PAGE = 512, 8, 2, 64, 16
E, K, F = 12, 4, 160


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def bf(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16).cuda()


def within_a_step(got, ref, what):
    ulps = bf16_ulps(f64(got), ref, floor=2.0 ** -10).max()
    assert ulps <= 1.0, f"{what}: {ulps:.2f} bf16 steps"


class Layer:
    def __init__(self, lib, b, seed):
        self.lib, self.b = lib, b
        g = torch.Generator().manual_seed(seed)
        lens = [1 + (37 * i) % 200 for i in range(b)]
        self.pw = W.build_prelude(b, H, HQ, HKV, D, seed=seed, lengths=lens, qk_norm=False, theta=1.0e4)
        self.aw = W.build(lens, HQ, HKV, D, PAGE, seed=seed + 1)
        self.x, self.w_qkv = bf(self.pw.x), lib.pack_weights(bf(self.pw.w_qkv))
        self.kc, self.vc = bf(self.aw.k_cache), bf(self.aw.v_cache)
        self.bt, self.cl = torch.from_numpy(self.aw.block_table).cuda(), torch.from_numpy(self.aw.context_lens).cuda()
        c = lambda *s, std=1.0, mean=0.0: values(g, *s, std=std, mean=mean).cuda()
        self.w_o, self.residual, self.norm_w = c(H, HQ * D, std=(HQ * D) ** -0.5), c(b, H), c(H, mean=1.0, std=0.1)
        # the router's rows, padded to 16: the last four are no experts
        self.w_router = c(16, H, std=2 * H ** -0.5)
        self.up, self.down = c(E, 2 * F, H, std=H ** -0.5), c(E, H, F, std=F ** -0.5)
        self.shared_up, self.shared_down = c(2 * F, H, std=H ** -0.5), c(H, F, std=F ** -0.5)
        self.post_w, self.pre_w = c(H, mean=1.0, std=0.1), c(H, mean=1.0, std=0.1)
        p = lib.pack_weights
        self.packed = dict(w_o=p(self.w_o), router=p(self.w_router), up=p(self.up.flatten(0, 1)).view(self.up.shape),
                           down=p(self.down.flatten(0, 1)).view(self.down.shape), shared_up=p(self.shared_up),
                           shared_down=p(self.shared_down))
        e = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device="cuda")
        self.q, self.attn, self.z, self.h = e(b, HQ, D), e(b, HQ, D), e(b, H), e(b, H)
        self.logits, self.ids, self.weights = e(b, 16, dt=torch.float32), e(b, K, dt=torch.int32), e(b, K, dt=torch.float32)
        self.inner, self.dense, self.out, self.z2, self.h2 = e(b, F), e(b, H), e(b, H), e(b, H), e(b, H)

    def step(self):
        lib, p = self.lib, self.packed
        lib.attention_prelude_append(self.x, self.w_qkv, self.cl, self.q, self.kc, self.vc, self.bt, num_q_heads=HQ,
                                     num_kv_heads=HKV, head_dim=D, rope_theta=1.0e4)
        lib.paged_decode_attention(self.q, self.kc, self.vc, self.bt, self.cl, self.attn, D ** -0.5)
        lib.o_proj_residual_norm(self.attn.view(self.b, HQ * D), p["w_o"], self.residual, self.norm_w, self.z, self.h)
        lib.linear(self.h, p["router"], self.logits)
        lib.moe_route(self.logits[:, :E], self.ids, self.weights, renormalise=True)
        # a shared expert, dense, then the chosen ones on top of it
        lib.linear(self.h, p["shared_up"], self.inner, activation="silu", gated=True)
        lib.linear(self.inner, p["shared_down"], self.dense)
        lib.moe_experts(self.h, self.ids, self.weights, p["up"], p["down"], self.out, residual=self.dense)
        lib.block_norm(self.out, self.z, self.z2, self.h2, post_w=self.post_w, pre_w=self.pre_w, eps=1e-6)

    def outputs(self):
        return [t.clone() for t in (self.q, self.attn, self.z, self.h, self.logits, self.ids, self.weights, self.inner,
                                    self.dense, self.out, self.z2, self.h2)]

    def check(self):
        rq, _, _ = oracle.prelude(self.pw.x, self.pw.w_qkv, HQ, HKV, D, self.pw.context_lens, 1.0e4)
        within_a_step(self.q, rq, "q")
        ra = oracle.attend(bits(self.q), bits(self.kc), bits(self.vc), self.aw.block_table, self.aw.context_lens, D ** -0.5)[0]
        within_a_step(self.attn, ra, "attention")
        rz, rh = oracle.o_proj_residual_norm(bits(self.attn.view(self.b, HQ * D)), bits(self.w_o), bits(self.residual),
                                             bits(self.norm_w), 1e-5)
        within_a_step(self.z, rz, "z")
        within_a_step(self.h, rh, "h")
        h = f64(self.h)
        ref = ffn.linear(h, f64(self.w_router))
        check(self.logits, ref, linear_error(h, f64(self.w_router), None, None, "none", False, ref, True), "router logits")
        ids, w = ffn.moe_route(f64(self.logits)[:, :E], K)
        assert np.array_equal(self.ids.cpu().numpy(), ids)
        assert (np.abs(f64(self.weights) - w) <= 1.01 * F32 * w + 2.0 ** -149).all()
        up, down = f64(self.shared_up), f64(self.shared_down)
        ref = ffn.linear(h, up, activation="silu", gated=True)
        check(self.inner, ref, linear_error(h, up, None, None, "silu", True, ref, False), "shared gate and up")
        ref = ffn.linear(f64(self.inner), down)
        check(self.dense, ref, linear_error(f64(self.inner), down, None, None, "none", False, ref, False), "shared down")
        s = dict(x=self.h, ids=self.ids.cpu(), weights=self.weights.cpu(), up=self.up, down=self.down, residual=self.dense)
        check(self.out, *experts_reference(s, "silu"), "experts")
        s = dict(y=self.out, residual=self.z, post_w=self.post_w, pre_w=self.pre_w, gate=None)
        (z, bz), (hn, bh) = norm_reference(s, 1.0, 0.0, 1e-6)
        check(self.z2, z, bz, "next residual")
        check(self.h2, hn, bh, "next input")


@pytest.mark.parametrize("b", [1, 5, 40, 100])
def test_a_layer_and_its_graph(gpu_lib, b):
    layer = Layer(gpu_lib, b, seed=20 + b)
    layer.step()
    torch.cuda.synchronize()
    layer.check()
    want = layer.outputs()
    # the largest of every kind reserved on the stream that captures
    s = torch.cuda.Stream()
    gpu_lib.workspace_reserve(b, HQ, HKV, D, PAGE, layer.bt.shape[1], stream=s)
    gpu_lib.prelude_workspace_reserve(gpu_lib.prelude_dims(b, H, HQ, HKV, D, D, False, 1e4, 1e-6), stream=s)
    gpu_lib.o_proj_workspace_reserve(b, HQ * D, H, stream=s)
    gpu_lib.linear_workspace_reserve(gpu_lib.linear_dims(b, H, 2 * F), stream=s)
    gpu_lib.linear_workspace_reserve(gpu_lib.linear_dims(b, H, F, "silu", True), stream=s)
    gpu_lib.linear_workspace_reserve(gpu_lib.linear_dims(b, F, H), stream=s)
    gpu_lib.moe_workspace_reserve(gpu_lib.moe_dims(b, H, F, E, K), stream=s)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        layer.step()
    for _ in range(3):
        for t in (layer.q, layer.attn, layer.z, layer.h, layer.logits, layer.weights, layer.inner, layer.dense, layer.out,
                  layer.z2, layer.h2):
            t.fill_(float("nan"))
        layer.ids.fill_(-5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(layer.outputs(), want):
            assert torch.equal(a, c)
        layer.step()  # eager, on the current stream, between replays
        torch.cuda.synchronize()
        for a, c in zip(layer.outputs(), want):
            assert torch.equal(a, c)
