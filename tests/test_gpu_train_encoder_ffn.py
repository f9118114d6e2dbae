"""examples/train_encoder.py with feed-forward blocks: the gradients of a step against float64 autograd of the same model.

Bound: as test_gpu_train_encoder.py has for two attentions and three norms, 5e-2 of a gradient's largest element and 3e-2 of its 2-norm
(two attentions, two feed-forward blocks and five norms: twice the stages, whose roundings add up in quadrature, sqrt(2)), and what the 8-bit
checkpoints add: x' and h' are off by up to half a step of a block of 32, 2^-8 to 2^-7 of its largest element, with the sign of chance; against
the rms of normal elements, whose largest of 32 is 2.1 of it, 2.1 * 2^-7.5 / sqrt(3) = 0.7e-2 a weight gradient and, through the derivative of
GELU, dh.  Together 8e-2 and 5e-2."""
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
    d = r.shape[-1]

    def layer_norm(t, k):
        return torch.nn.functional.layer_norm(t, (d,), p["w%d" % k], p["b%d" % k], 1e-5)

    h = layer_norm(r, 0)
    for k, kind in enumerate(enc.blocks):
        if kind == "attention":
            q, key, v = (torch.stack((h @ p["%s%d" % (name, k)]).split(d // H, -1), 1) for name in ("Wq", "Wk", "Wv"))
            a = torch.softmax(q @ key.transpose(-1, -2) / (d // H) ** 0.5, -1) @ v
            f = torch.cat(a.unbind(1), -1) @ p["Wo%d" % k]
        else:
            f = torch.nn.functional.gelu(h @ p["W1%d" % k] + p["b1%d" % k]) @ p["W2%d" % k] + p["b2%d" % k]
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
    enc = ex.Encoder(ctx, B, L, N, d, H, 2, seed=5, ffn=192)
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
        assert err.max() <= 8e-2 * np.abs(want[k]).max(), (k, err.max() / np.abs(want[k]).max())
        assert np.linalg.norm(err) <= 5e-2 * np.linalg.norm(want[k]), (k, np.linalg.norm(err) / np.linalg.norm(want[k]))


def test_it_trains():
    losses = ex.train(steps=20, ffn=256)
    assert len(losses) == 20 and np.isfinite(losses).all()
