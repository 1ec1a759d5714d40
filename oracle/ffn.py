"""fp64 reference of the feed-forward half of a decode layer: a product with
its epilogue, routing, the experts' products and the block norms.  Written
from the definitions in include/pda.h, in NumPy, apart from the library and
from perf/.  Arrays are float64 values (bf16 inputs as what they stand for)."""
from __future__ import annotations

import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activate(x, name):
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "silu":
            y = x / (1.0 + np.exp(-x))
        elif name == "gelu":
            y = 0.5 * x * _erfc(-x / math.sqrt(2.0))  # 1 + erf(z), without its cancellation at z < 0
        elif name == "gelu_tanh":
            y = x / (1.0 + np.exp(-math.sqrt(8.0 / math.pi) * (x + 0.044715 * x ** 3)))  # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
        elif name == "relu":
            y = np.where(np.isnan(x), x, np.maximum(x, 0.0))
        else:
            assert name == "none"
            return x
    return np.where(x == -np.inf, 0.0, y)  # the limit


def linear(x, w, bias=None, residual=None, activation="none", gated=False):
    """x [B, K], w [N, K] (gated: [2 N, K], the gate's rows first) -> [B, N]."""
    y = x @ w.T
    if bias is not None:
        y = y + bias
    if gated:
        n = w.shape[0] // 2
        y = activate(y[:, :n], activation) * y[:, n:]
    else:
        y = activate(y, activation)
    return y if residual is None else y + residual


def moe_route(logits, top_k, scoring="softmax", renormalise=True, select_bias=None, scale=1.0):
    """Experts [T, top_k] and weights [T, top_k], a token and a choice at a time."""
    most = float(np.finfo(np.float32).max)
    ids = np.zeros((logits.shape[0], top_k), dtype=np.int32)
    weights = np.zeros(ids.shape)
    for t, row in enumerate(np.asarray(logits, dtype=np.float64)):
        allowed = ~np.isnan(row) & (row != -np.inf)
        l = np.where(allowed, np.minimum(row, most), 0.0)
        if not allowed.any():
            score = np.zeros(l.size)
        elif scoring == "softmax":
            e = np.where(allowed, np.exp(l - l[allowed].max()), 0.0)
            score = e / e.sum()
        else:
            with np.errstate(over="ignore"):
                score = np.where(allowed, 1.0 / (1.0 + np.exp(-l)), 0.0)
        key = l if select_bias is None else score + np.asarray(select_bias, dtype=np.float64)
        order = sorted(range(l.size), key=lambda e: (not allowed[e], -key[e] if allowed[e] else 0.0, e))
        ids[t] = order[:top_k]
        w = score[ids[t]]
        if renormalise:
            w = w / w.sum() if w.sum() > 0 else np.zeros(top_k)
        weights[t] = w * scale
    return ids, weights


def moe_experts(x, ids, weights, w_gate_up, w_down, residual=None, activation="silu", hidden=None):
    """x [T, H], ids and weights [T, top_k], w_gate_up [E, 2 F, H], w_down [E, H, F] -> [T, H].  ``hidden``, a
    dict, takes each pair's act(G x) * (U x) by (t, j)."""
    e_count, _, f = w_down.shape
    out = np.zeros(x.shape) if residual is None else residual.astype(np.float64)
    for t in range(x.shape[0]):
        for j in range(ids.shape[1]):
            e = int(ids[t, j])
            if not 0 <= e < e_count:
                continue
            h = activate(w_gate_up[e, :f] @ x[t], activation) * (w_gate_up[e, f:] @ x[t])
            if hidden is not None:
                hidden[t, j] = h
            out[t] = out[t] + float(weights[t, j]) * (w_down[e] @ h)
    return out


def block_norm(y, residual=None, post_w=None, pre_w=None, gate=None, scale=1.0, weight_offset=0.0, eps=1e-5):
    """z [R, H], and h [R, H] or None."""
    def norm(v, w):
        with np.errstate(divide="ignore", invalid="ignore"):
            return v / np.sqrt(np.mean(v * v, axis=1, keepdims=True) + eps) * (w + weight_offset)

    u = y if post_w is None else norm(y, post_w)
    u = u if gate is None else u * gate
    z = scale * u if residual is None else residual + scale * u
    return z, (None if pre_w is None else norm(z, pre_w))
