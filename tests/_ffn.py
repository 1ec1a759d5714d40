"""Helpers for the tests of the feed-forward operators."""
import numpy as np
import torch

HALF = 2.0 ** -8    # half a bf16 step, relative to the value
F32 = 2.0 ** -24    # the same of fp32
TINY = 2.0 ** -133  # bf16's smallest number


def values(g, *shape, std=1.0, mean=0.0):
    """bf16 normal values on the host."""
    return (torch.randn(*shape, generator=g) * std + mean).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().double().numpy()


def gpu(t):
    return None if t is None else t.cuda()


def chain(k):
    """Roundings in a row in an fp32 sum of k products on the matrix cores: the products of a 32-long
    step one after the other, then a step at a time, then at most 16 partial sums."""
    return 32 + k // 32 + 16


def sum_error(x, w, bias=None):
    """Bound of the error of fp32 sums x w^T + bias: each rounding on the way is at most a step of a
    partial sum (a whole one, as the matrix cores may cut), which the sum of magnitudes bounds."""
    s = np.abs(x) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    return 2 * F32 * chain(x.shape[1]) * s


# The largest slope of an activation (gelu's forms reach 1.13) and its own error relative to its value, in
# fp32 steps: the exponential's argument is rounded (|z| up to 88 where its result matters: 0.5 |z| steps
# near 8, where the value has fallen to 2^-11 of its argument, and far below a bf16 step everywhere),
# reciprocal, products and erfc's few steps.
SLOPE = 1.13


def activation_error(x, y, err):
    """Error of act(x) = y when x is off by err."""
    return SLOPE * err + 16 * F32 * np.abs(y) + 16 * F32 * np.abs(x) * np.exp(-np.maximum(-x, 0.0) / 2)


def linear_error(x, w, bias, residual, activation, gated, out, f32):
    """Bound of |got - out| of a linear product whose fp64 value is ``out``."""
    from oracle import ffn
    pre = x @ w.T + (0.0 if bias is None else bias)
    err = sum_error(x, w, bias)
    if gated:
        n = w.shape[0] // 2
        g, u = pre[:, :n], pre[:, n:]
        a = ffn.activate(g, activation)
        ea = activation_error(g, a, err[:, :n]) if activation != "none" else err[:, :n]
        e = np.abs(a) * err[:, n:] + np.abs(u) * ea + ea * err[:, n:] + 2 * F32 * np.abs(a * u)
    else:
        a = ffn.activate(pre, activation)
        e = activation_error(pre, a, err) if activation != "none" else err
    if residual is not None:
        e = e + F32 * np.abs(out)
    return e + (F32 if f32 else HALF) * (np.abs(out) + e) + TINY


def check(got, ref, bound, what):
    got = got if isinstance(got, np.ndarray) else f64(got)
    assert got.shape == ref.shape, what
    assert np.isfinite(got).all(), f"{what}: not finite"
    ratio = np.abs(got - ref) / bound
    print(f"  {what}: worst error {ratio.max() if ratio.size else 0.0:.2f} of its bound (n={got.size})", flush=True)
    assert (ratio <= 1.0).all(), f"{what}: {ratio.max():.2f} of the bound at {np.unravel_index(ratio.argmax(), ratio.shape)}"
