"""examples/train_encoder.py: its gradients against float64 autograd of the same model, and a training run.

Bound of a gradient: a bf16 attention of this library is within 2e-2 of its largest element (util_gpu.TOL); here two of them and
three norms follow each other, whose rounding adds up: 5e-2 of the largest element of a gradient, and 3e-2 of its 2-norm.
"""
import numpy as np
import pytest
import torch

import examples.train_encoder as ex

pytestmark = pytest.mark.gpu


def reference(enc, x, sel, target, H):
    """Loss and gradients of the model in float64 on the CPU, weights as the kernels read them."""
    p = {k: t.double().cpu().requires_grad_() for k, t in enc.low.items()}
    z = x[:, sel.long()].double().cpu()
    z = (z - z.mean(-1, keepdim=True)) / z.var(-1, unbiased=False, keepdim=True).sqrt()
    r = z @ p["We"] + p["be"]
    B, n, d = r.shape

    def layer_norm(t, k):
        return torch.nn.functional.layer_norm(t, (d,), p["w%d" % k], p["b%d" % k], 1e-5)

    h = layer_norm(r, 0)
    for k in range(enc.layers):
        q, key, v = (torch.stack((h @ p["%s%d" % (name, k)]).split(d // H, -1), 1) for name in ("Wq", "Wk", "Wv"))
        a = torch.softmax(q @ key.transpose(-1, -2) / (d // H) ** 0.5, -1) @ v
        f = torch.cat(a.unbind(1), -1) @ p["Wo%d" % k]
        u = f / (f.square().mean(-1, keepdim=True) + 1e-5).sqrt() * p["wp%d" % k]
        r = ex.RES_SCALE * r + ex.BRANCH_SCALE * p["gate%d" % k] * u
        h = layer_norm(r, k + 1)
    loss = (h - target).square().mean()
    loss.backward()
    return float(loss.detach()), {k: t.grad.numpy() for k, t in p.items()}


def test_gradients_of_a_step():
    import paper_2501_14183_amd as vd
    ctx = vd.Context(0)
    B, N, L, d, H = 4, 40, 96, 128, 2
    enc = ex.Encoder(ctx, B, L, N, d, H, 2, seed=5)
    x = ex.windows(B, N, L, seed=1)
    sel = torch.tensor([0, 3, 4, 9, 17, 21, 22, 30, 31, 38, 39], dtype=torch.int32, device="cuda")
    n = len(sel)
    full = torch.zeros(N, dtype=torch.int32, device="cuda")
    full[:n] = sel
    n_dev = torch.tensor([n], dtype=torch.int32, device="cuda")
    target = torch.randn(B, n, d, generator=torch.Generator().manual_seed(3))
    packed = torch.zeros(B, N, d, device="cuda")
    packed.view(-1)[:target.numel()] = target.cuda().reshape(-1)
    loss, dh = ex.loss_and_gradient(enc.forward(x, full, n_dev), packed, n_dev, B)
    enc.backward(dh, n_dev)
    want_loss, want = reference(enc, x, sel, target.double(), H)
    assert abs(float(loss) - want_loss) <= 1e-2 * want_loss
    for k, g in enc.grads.items():
        g = g.double().cpu().numpy()
        if not np.abs(want[k]).max() > 0:
            continue
        err = np.abs(g - want[k])
        assert err.max() <= 5e-2 * np.abs(want[k]).max(), k
        assert np.linalg.norm(err) <= 3e-2 * np.linalg.norm(want[k]), k


def test_training_lowers_the_loss():
    losses = ex.train(steps=120)
    first, last = np.mean(losses[:10]), np.mean(losses[-10:])
    assert np.isfinite(losses).all() and last < 0.5 * first, (first, last)
