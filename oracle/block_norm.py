"""Norms before and after a block with its gate and the residual scale, forward and backward, in fp64.  Test infrastructure.

    u = post(f),  r = alpha x + beta g * u,  h = pre(r)

post and pre are "none", "layer" ((v - mean) / sqrt(var + eps), population variance) or "rms" (v / sqrt(mean(v^2) + eps)), each
with an optional weight and bias; g is None, one row [d] or a row for every window [B, d].  `stats` holds the mean and
1 / deviation of post and of pre for every token, 0 and 1 where there is no norm, mean 0 for "rms".
"""
import numpy as np

KINDS = ("none", "layer", "rms")


def _f64(a):
    return None if a is None else np.asarray(a, dtype=np.float64)


def moments(kind, v, eps):
    """(mean, 1 / deviation) of every row of v [..., d]."""
    mean, inv = np.zeros(v.shape[:-1]), np.ones(v.shape[:-1])
    for at in np.ndindex(*v.shape[:-1]):
        row = v[at]
        if kind == "layer":
            mean[at] = row.sum() / row.size
        if kind != "none":
            inv[at] = 1.0 / np.sqrt(((row - mean[at]) ** 2).sum() / row.size + eps)
    return mean, inv


def gate_rows(gate, B, d):
    gate = _f64(gate)
    return np.ones((B, 1, d)) if gate is None else np.broadcast_to(gate.reshape(-1, 1, d), (B, 1, d))


def block_norm_forward(x, f=None, pre="layer", w=None, b=None, post="none", wp=None, bp=None, gate=None, alpha=1.0, beta=1.0,
                       eps=1e-5):
    """x, f [B, n, d] -> (r, h, stats [B, n, 4]); h is None when pre is "none"."""
    x, f, w, b, wp, bp = map(_f64, (x, f, w, b, wp, bp))
    B, n, d = x.shape
    stats = np.zeros((B, n, 4))
    stats[..., 1] = 1.0
    r = alpha * x
    if f is not None:
        mean, inv = moments(post, f, eps)
        stats[..., 0], stats[..., 1] = mean, inv
        u = (f - mean[..., None]) * inv[..., None]
        if wp is not None:
            u = u * wp
        if bp is not None:
            u = u + bp
        r = r + beta * gate_rows(gate, B, d) * u
    mean, inv = moments(pre, r, eps)
    stats[..., 2], stats[..., 3] = mean, inv
    if pre == "none":
        return r, None, stats
    h = (r - mean[..., None]) * inv[..., None]
    if w is not None:
        h = h * w
    if b is not None:
        h = h + b
    return r, h, stats


def _norm_backward(kind, dhat, hat, inv):
    """Gradient of a norm's input from that of the normalised row: the derivative of (v - mean(v)) / deviation(v)."""
    if kind == "none":
        return dhat
    out = dhat - hat * (dhat * hat).mean(-1, keepdims=True)
    if kind == "layer":
        out = out - dhat.mean(-1, keepdims=True)
    return inv[..., None] * out


def block_norm_backward(dr, dh, r, f, stats, pre="layer", w=None, post="none", wp=None, bp=None, gate=None, alpha=1.0, beta=1.0):
    """Gradients of sum(r * dr) + sum(h * dh), as a dict: dx, df, dw, db, dwp, dbp, dgate."""
    dr, dh, r, f, stats, w, wp, bp = map(_f64, (dr, dh, r, f, stats, w, wp, bp))
    like = r if dr is None else dr
    B, n, d = like.shape
    D = np.zeros(like.shape) if dr is None else dr.copy()
    out = {}
    if pre != "none":
        hat = (r - stats[..., 2:3]) * stats[..., 3:4]
        out["db"], out["dw"] = dh.sum((0, 1)), (dh * hat).sum((0, 1))
        D = D + _norm_backward(pre, dh if w is None else dh * w, hat, stats[..., 3])
    out["dx"] = alpha * D
    g = gate_rows(gate, B, d)
    du = beta * g * D
    if f is None:
        out["df"] = du
        return out
    hat = (f - stats[..., 0:1]) * stats[..., 1:2]
    u = hat if wp is None else hat * wp
    u = u if bp is None else u + bp
    out["dbp"], out["dwp"] = du.sum((0, 1)), (du * hat).sum((0, 1))
    if gate is not None:
        dg = (beta * D * u).sum(1)
        out["dgate"] = dg if np.ndim(gate) == 2 and len(gate) == B else dg.sum(0).reshape(np.shape(gate))
    out["df"] = _norm_backward(post, du if wp is None else du * wp, hat, stats[..., 1])
    return out
