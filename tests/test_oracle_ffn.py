"""The feed-forward oracle against closed forms and hand-worked cases."""
import math

import numpy as np
import pytest

from oracle import ffn


def test_activations_at_known_points():
    x = np.array([-np.inf, -1.0, 0.0, 1.0, np.inf])
    assert np.allclose(ffn.activate(x, "silu")[1:4], [-1 / (1 + math.e), 0.0, 1 / (1 + 1 / math.e)])
    assert np.allclose(ffn.activate(x, "gelu")[1:4], [-0.15865525393145707, 0.0, 0.8413447460685429])
    assert np.allclose(ffn.activate(x, "gelu_tanh")[1:4], [-0.15880800939172324, 0.0, 0.8411919906082768])
    for name in ("silu", "gelu", "gelu_tanh", "relu"):
        y = ffn.activate(x, name)
        assert y[0] == 0.0 and y[4] == np.inf
    assert math.isnan(ffn.activate(np.array([np.nan]), "relu")[0])


def test_linear_is_its_rows():
    x, w = np.array([[1.0, 2.0]]), np.array([[1.0, 0.0], [0.0, 1.0], [1.0, 1.0], [-1.0, 1.0]])
    assert ffn.linear(x, w).tolist() == [[1.0, 2.0, 3.0, 1.0]]
    assert ffn.linear(x, w, bias=np.array([0.0, 0.0, 0.0, -2.0]), activation="relu").tolist() == [[1.0, 2.0, 3.0, 0.0]]
    assert ffn.linear(x, w, residual=np.array([[10.0, 20.0]]), gated=True).tolist() == [[13.0, 22.0]]


def test_route_orders_masks_and_ties():
    inf = np.inf
    ids, w = ffn.moe_route(np.array([[0.0, math.log(3.0), -inf, 0.0]]), 3, renormalise=False)
    assert ids.tolist() == [[1, 0, 3]] and np.allclose(w, [[0.6, 0.2, 0.2]])
    ids, w = ffn.moe_route(np.array([[0.0, math.log(3.0), -inf, 0.0]]), 4, scale=2.0)
    assert ids.tolist() == [[1, 0, 3, 2]] and np.allclose(w, [[1.2, 0.4, 0.4, 0.0]])
    ids, w = ffn.moe_route(np.array([[-inf, np.nan, -inf]]), 2, scoring="sigmoid")
    assert ids.tolist() == [[0, 1]] and w.tolist() == [[0.0, 0.0]]
    ids, w = ffn.moe_route(np.array([[inf, 1.0, inf]]), 3)
    assert ids.tolist() == [[0, 2, 1]] and np.allclose(w, [[0.5, 0.5, 0.0]])
    ids, w = ffn.moe_route(np.array([[0.0, 0.0, 5.0]]), 1, scoring="sigmoid", select_bias=np.array([0.0, 2.0, 0.0]),
                           renormalise=False)
    assert ids.tolist() == [[1]] and w.tolist() == [[0.5]]


def test_experts_are_gated_products():
    x = np.array([[1.0, -2.0]])
    up = np.array([[[1.0, 0.0], [0.0, 1.0]], [[0.0, -1.0], [2.0, 0.0]]])  # E 2, F 1: G, U
    down = np.array([[[1.0], [10.0]], [[100.0], [0.0]]])
    got = ffn.moe_experts(x, np.array([[0, 1]]), np.array([[0.5, 2.0]]), up, down, activation="none")
    # expert 0: 1 * -2 = -2; expert 1: 2 * 2 = 4
    assert got.tolist() == [[0.5 * -2 + 2 * 400.0, 0.5 * -20.0]]
    none = ffn.moe_experts(x, np.array([[-1, 2]]), np.ones((1, 2)), up, down, residual=np.array([[3.0, 4.0]]))
    assert none.tolist() == [[3.0, 4.0]]


@pytest.mark.parametrize("offset", [0.0, 1.0])
def test_block_norm_by_hand(offset):
    y, res = np.array([[3.0, 4.0]]), np.array([[1.0, 0.0]])
    rms = math.sqrt(12.5)
    z, h = ffn.block_norm(y, res, post_w=np.ones(2) - offset, pre_w=np.ones(2) - offset, gate=np.array([2.0, 1.0]),
                          scale=0.5, weight_offset=offset, eps=0.0)
    want = np.array([[1.0 + 3.0 / rms, 2.0 / rms]])
    assert np.allclose(z, want) and np.allclose(h, want / math.sqrt((want ** 2).mean()))
    z, h = ffn.block_norm(y)
    assert z.tolist() == y.tolist() and h is None
