"""Inputs of the feed-forward block's GPU tests, and how far its results may be off (not a test module).

u = 2^-24 is the error of one fp32 operation.  A sum of K products is off by at most (K + 4) 2 u times the sum of their magnitudes,
in any order (a product of three-part numbers by itself: 2 u); GELU and its derivative have slopes of at most 1.13 and 0.8 and are
themselves off by 8 u of their magnitude.  In the bf16 form a fitted Q = 1 - Phi(|x|) is off by 2.7e-5 of itself and by 16 u (a polynomial of
degree 6 and the exponential; its argument of up to 25 costs 25 * 7 u more), and S = Q - |x| phi by 1.5e-5 beside that; from |x| = 5.5 on
both are held, which is off by 1.1e-7 and 6e-7.  test_ffn_host.py evaluates the fits.  A rounding to bf16 is off by at most 2^-8 of the value.  These are followed through the block.
"""
import numpy as np

import workloads as wl
from oracle import feedforward as o

U, BF = 2.0 ** -24, 2.0 ** -8


def product_error(A, B, eA=0.0, eB=0.0):
    """Magnitude of the error of A @ B in fp32 with operands off by eA, eB."""
    A, B = np.abs(A), np.abs(B)
    return A @ B * ((A.shape[-1] + 4) * 2 * U) + (eA @ (B + eB) if np.ndim(eA) else 0.0) + (A @ eB if np.ndim(eB) else 0.0)


def act_error(x, ex, dtype, act, slope=False):
    """Error of act(x), or of its derivative, for x off by ex."""
    ex = ex + 0.0 * x
    if act == "relu":
        return 0.0 * x if slope else ex
    if dtype == "fp32":
        own = 8 * U * (1 + np.abs(x))
    else:
        tail = o.cdf(-np.abs(x)) * (2.7e-5 + 200 * U)
        own = (tail + 1.5e-5 + 6e-7 if slope else np.abs(x) * tail + 1.1e-7) + 8 * U * (1 + np.abs(x))
    return own + (0.8 if slope else 1.13) * ex


def rounded(x, ex, dtype):
    return ex if dtype == "fp32" else ex + BF * (np.abs(x) + ex)


def make(seed, B, n, d, f, dtype, bias=True):
    rng = np.random.default_rng([0xFF, seed, B, n, d, f])
    q = lambda a: wl.quantise(a, dtype)
    t = dict(x=q(rng.standard_normal((B * n, d)) * (0.4 + rng.standard_normal(d) ** 2) + 0.3), dy=q(rng.standard_normal((B * n, d))),
             W1=q(rng.standard_normal((d, f)) / d ** 0.5), W2=q(rng.standard_normal((f, d)) / f ** 0.5),
             b1=q(0.2 * rng.standard_normal(f)) if bias else None, b2=q(0.2 * rng.standard_normal(d)) if bias else None)
    return t


def forward_bounds(t, dtype, act):
    """(y, its bound, h, its bound)."""
    y, h = o.forward(t["x"], t["W1"], t["b1"], t["W2"], t["b2"], act)
    eh = product_error(t["x"], t["W1"]) + 2 * U * (np.abs(h) + (0 if t["b1"] is None else np.abs(t["b1"])))
    a = o.activation(act, h)
    ea = rounded(a, act_error(h, eh, dtype, act), dtype)
    ey = product_error(a, t["W2"], ea) + 2 * U * (np.abs(y) + (0 if t["b2"] is None else np.abs(t["b2"])))
    return y, rounded(y, ey, dtype), h, eh


def backward_bounds(t, x, h, dtype, act, grad="fp32"):
    """{name: (value, bound)} from the x and h that the checkpoints stand for."""
    want = o.backward(t["dy"], x, h, t["W1"], t["W2"], act)
    da, rise, a = t["dy"] @ t["W2"].T, o.slope(act, h), o.activation(act, h)
    edh = product_error(t["dy"], t["W2"].T) * (np.abs(rise) + U) + np.abs(da) * act_error(h, 0.0, dtype, act, slope=True) + 2 * U * np.abs(want["dh"])
    edh = rounded(want["dh"], edh, dtype)
    ea = rounded(a, act_error(h, 0.0, dtype, act), dtype)
    T = x.shape[0]
    e = dict(dx=rounded(want["dx"], product_error(want["dh"], t["W1"].T, edh), dtype), dW1=product_error(x.T, want["dh"], 0.0, edh),
             dW2=product_error(a.T, t["dy"], ea.T), db1=edh.sum(0) + 2 * T * U * np.abs(want["dh"]).sum(0), db2=2 * T * U * np.abs(t["dy"]).sum(0))
    return {k: (want[k], e[k] if k == "dx" else rounded(want[k], e[k], grad)) for k in e}


def assert_within(name, got, want, bound):
    got = got.detach().double().cpu().numpy().reshape(want.shape)
    assert np.isfinite(got).all(), "%s: not finite" % name
    if not got.size:
        return
    over = np.abs(got - want) - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, "%s at %s: %.9g for %.9g, bound %.3g" % (name, at, got[at], want[at], bound[at])
    norm = np.sqrt((want ** 2).sum())
    off = np.sqrt(((got - want) ** 2).sum())
    # (bounds add up magnitudes; roundings of either sign stay far below them: two of 2^-8, whose mean square is a third, in quadrature)
    assert off <= 2.0 ** -7 * norm + np.sqrt((np.minimum(bound, 1e-30) ** 2).sum()), "%s: off by %.3g of its norm" % (name, off / norm)
