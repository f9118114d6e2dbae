"""examples/train_encoder.py with more than ten blocks: it runs, and a step writes the gradient of every weight."""
import numpy as np
import pytest
import torch

import examples.train_encoder as ex

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,ffn", [(64, 128), (64, 64)])
def test_every_gradient_is_written(d, ffn):
    import paper_2501_14183_amd as vd
    ctx = vd.Context(0)
    B, N, L, layers = 2, 24, 48, 6
    enc = ex.Encoder(ctx, B, L, N, d, 1, layers, seed=5, ffn=ffn)
    assert len(enc.blocks) == 12
    x, sel = ex.windows(B, N, L, seed=1), torch.arange(N, dtype=torch.int32, device="cuda")
    n_dev = torch.tensor([N - 3], dtype=torch.int32, device="cuda")
    target = torch.randn(B, N, d, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    for g in enc.grads.values():
        g.fill_(float("nan"))
    loss, dh = ex.loss_and_gradient(enc.forward(x, sel, n_dev), target, n_dev, B)
    enc.backward(dh, n_dev)
    assert bool(torch.isfinite(loss))
    for k, g in enc.grads.items():
        assert bool(torch.isfinite(g).all()) and bool(g.any()), k


def test_it_runs():
    losses = ex.train(steps=3, layers=6, ffn=192)
    assert len(losses) == 3 and np.isfinite(losses).all()
