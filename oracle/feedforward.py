"""The feed-forward block, its 8-bit checkpoints and 8-bit integer products, in fp64.  Test infrastructure.

pack8 / unpack8: rows in blocks of 32 channels, whole numbers of -127..127 times the smallest power of two (at least 2^-126) with which
the block's largest magnitude is, rounded, at most 127; ties to even.  An exponent byte of 255 marks a block with an infinity or NaN.
"""
import math

import numpy as np

BLOCK = 32
ACTS = ("none", "relu", "gelu")


def pack8(x):
    """x [rows, d] -> (codes int8 [rows, d], exponent bytes [rows, ceil(d / 32)])."""
    x = np.asarray(x, dtype=np.float64)
    rows, d = x.shape
    nb = -(-d // BLOCK)
    codes, exps = np.zeros((rows, d), dtype=np.int8), np.zeros((rows, nb), dtype=np.uint8)
    for r in range(rows):
        for b in range(nb):
            part = x[r, b * BLOCK:(b + 1) * BLOCK]
            if not np.isfinite(part).all():
                exps[r, b] = 255
                continue
            most, e = np.abs(part).max(), -126
            if most > 0.0:
                e = max(math.frexp(most)[1] - 7, -126)
                if np.rint(math.ldexp(most, -e)) > 127:
                    e += 1
            e = min(e, 121)
            exps[r, b] = e + 127
            codes[r, b * BLOCK:(b + 1) * BLOCK] = np.clip(np.rint(np.ldexp(part, -e)), -127, 127)
    return codes, exps


def unpack8(codes, exps):
    d = codes.shape[1]
    step = np.where(exps == 255, np.nan, np.ldexp(1.0, exps.astype(np.int64) - 127))
    return codes * np.repeat(step, BLOCK, axis=1)[:, :d]


def through_8_bits(x):
    return unpack8(*pack8(np.reshape(x, (-1, np.shape(x)[-1])))).reshape(np.shape(x))


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def cdf(x):
    return 0.5 * _erfc(-x / math.sqrt(2.0))


def activation(kind, x):
    if kind == "none":
        return x
    return np.where(x < 0, 0.0, x) if kind == "relu" else x * cdf(x)


def slope(kind, x):
    if kind == "relu":
        return (x > 0).astype(np.float64)
    return cdf(x) + x * np.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)


def forward(x, W1, b1, W2, b2, act):
    """x [T, d] -> (y, h)."""
    h = x @ W1 + (0.0 if b1 is None else b1)
    return activation(act, h) @ W2 + (0.0 if b2 is None else b2), h


def backward(dy, x, h, W1, W2, act):
    """Gradients from the x and h that are at hand -> dict."""
    dh = (dy @ W2.T) * slope(act, h)
    return dict(dx=dh @ W1.T, dW1=x.T @ dh, dW2=activation(act, h).T @ dy, db1=dh.sum(0), db2=dy.sum(0), dh=dh)


def integers(x):
    """Rows of fp32 numbers -> (codes int8, scale fp32): fp32 operations, each rounded once."""
    x = np.asarray(x, dtype=np.float32)
    most = np.abs(x).max(axis=1)
    codes, scale = np.zeros(x.shape, dtype=np.int8), np.zeros(x.shape[0], dtype=np.float32)
    for r, m in enumerate(most):
        if not np.isfinite(m):
            scale[r] = np.nan
        elif m >= np.float32(2.0 ** -100):
            scale[r] = m / np.float32(127)
            codes[r] = np.rint(x[r] * (np.float32(127) * (np.float32(1) / m)))
    return codes, scale


def linear_i8(x, W, bias, act):
    """act(x W + bias) from 8-bit integers, x [T, K], W [K, N]."""
    q, s = integers(x)
    w, c = integers(np.ascontiguousarray(np.asarray(W).T))
    y = (q.astype(np.int64) @ w.astype(np.int64).T) * (s.astype(np.float64)[:, None] * c.astype(np.float64)[None, :])
    return activation(act, y + (0.0 if bias is None else bias))
