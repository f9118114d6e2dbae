"""Pins of oracle/block_norm.py: closed forms, torch's norms in fp64, and its gradients against central differences."""
import itertools

import numpy as np
import pytest
import torch

from oracle import block_norm as o


def inputs(seed, B=2, n=3, d=5):
    rng = np.random.default_rng([0xB10C, seed, B, n, d])
    v = lambda *s: rng.standard_normal(s)
    return dict(x=v(B, n, d) + 0.5, f=v(B, n, d) - 0.3, w=1 + 0.2 * v(d), b=0.1 * v(d), wp=1 + 0.2 * v(d), bp=0.1 * v(d),
                shared=v(d), window=v(B, d)), v(B, n, d), v(B, n, d)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_is_torchs(kind):
    t, _, _ = inputs(0, d=7)
    r, h, stats = o.block_norm_forward(t["x"], pre=kind, w=t["w"], b=t["b"], eps=1e-3)
    x, w, b = (torch.from_numpy(t[k]) for k in ("x", "w", "b"))
    want = torch.nn.functional.layer_norm(x, (7,), w, b, 1e-3) if kind == "layer" else x / (x.square().mean(-1, keepdim=True) + 1e-3).sqrt() * w + b
    assert np.array_equal(r, t["x"])
    assert np.allclose(h, want.numpy(), rtol=1e-13, atol=1e-13)


def test_constant_and_known_rows():
    r, h, stats = o.block_norm_forward(np.full((1, 1, 4), 3.0), pre="layer", eps=1e-5)
    assert np.array_equal(h, np.zeros((1, 1, 4))) and stats[0, 0, 2] == 3.0 and np.isclose(stats[0, 0, 3], 1e5 ** 0.5)
    r, h, stats = o.block_norm_forward(np.array([[[3.0, 4.0]]]), pre="rms", eps=1e-30)
    assert np.allclose(h, np.array([3.0, 4.0]) / 12.5 ** 0.5)
    # residual scale, branch scale and gate: r = 2 x + 3 g f
    r, h, stats = o.block_norm_forward(np.ones((2, 1, 2)), np.full((2, 1, 2), 5.0), pre="none", gate=np.array([[1.0, 0.0], [0.0, -1.0]]),
                                       alpha=2.0, beta=3.0)
    assert h is None and np.array_equal(r, np.array([[[17.0, 2.0]], [[2.0, -13.0]]]))


@pytest.mark.parametrize("pre,post,gate", itertools.product(o.KINDS, o.KINDS, ("none", "shared", "window")))
def test_gradients_against_central_differences(pre, post, gate):
    """Differences of step 1e-6: error of order 1e-12 / 1e-6 from rounding and 1e-12 from the third derivative."""
    t, dr, dh = inputs(1)
    names = ["x", "f"] + (["w", "b"] if pre != "none" else []) + (["wp", "bp"] if post != "none" else [])
    args = {k: t[k] for k in names}
    if gate != "none":
        args["gate"] = t[gate]
    kw = dict(pre=pre, post=post, alpha=0.7, beta=-1.3, eps=1e-2)

    def loss(a):
        r, h, _ = o.block_norm_forward(**a, **kw)
        return (r * dr).sum() + (0.0 if h is None else (h * dh).sum())

    r, h, stats = o.block_norm_forward(**args, **kw)
    got = o.block_norm_backward(dr, None if pre == "none" else dh, r, t["f"], stats, pre=pre, w=args.get("w"), post=post,
                                wp=args.get("wp"), bp=args.get("bp"), gate=args.get("gate"), alpha=0.7, beta=-1.3)
    for name, a in args.items():
        want = np.zeros(a.shape)
        for at in np.ndindex(*a.shape):
            step = np.zeros(a.shape)
            step[at] = 1e-6
            want[at] = (loss({**args, name: a + step}) - loss({**args, name: a - step})) / 2e-6
        assert np.abs(got["d" + name] - want).max() <= 1e-7 * max(1.0, np.abs(want).max()), name


def test_shared_gate_of_shape_1_d_keeps_its_shape():
    t, dr, dh = inputs(2, B=3)
    r, h, stats = o.block_norm_forward(t["x"], t["f"], gate=t["shared"][None])
    g = o.block_norm_backward(dr, dh, r, t["f"], stats, gate=t["shared"][None])
    assert g["dgate"].shape == (1, 5)
