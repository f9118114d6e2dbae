"""Pins of oracle/optimiser.py: hand-computed values and torch's AdamW in fp64."""
import numpy as np
import torch

from oracle import optimiser as o


def test_norm_and_factor_by_hand():
    assert o.grad_norm([np.array([3.0]), np.zeros((0,)), np.array([[0.0, 4.0]])]) == 5.0
    assert o.grad_norm([]) == 0.0
    assert o.clip_factor(5.0, 10.0) == 1.0 and o.clip_factor(5.0, 0.0) == 1.0
    assert np.isclose(o.clip_factor(5.0, 1.0), 1.0 / 5.000001, rtol=1e-15)


def test_first_step_moves_by_the_rate():
    """From zero moments m / (1 - b1) = g and sqrt(v / (1 - b2)) = |g|: the step is lr sign(g) but for eps."""
    p, m, v = o.adamw(np.array([1.0, -2.0, 0.0]), np.zeros(3), np.zeros(3), np.array([0.5, -3.0, 0.0]), 0.1, 1, eps=1e-30)
    assert np.allclose(p, [0.9, -1.9, 0.0], rtol=1e-14)
    assert np.allclose(m, [0.05, -0.3, 0.0]) and np.allclose(v, [0.00025, 0.009, 0.0])


def test_steps_are_torchs():
    rng = np.random.default_rng(7)
    p = rng.standard_normal(50)
    t = torch.nn.Parameter(torch.from_numpy(p.copy()))
    opt = torch.optim.AdamW([t], lr=0.01, betas=(0.8, 0.99), eps=1e-6, weight_decay=0.1)
    m = v = np.zeros(50)
    for step in range(1, 6):
        g = rng.standard_normal(50)
        t.grad = torch.from_numpy(g.copy())
        norm = float(torch.nn.utils.clip_grad_norm_([t], 3.0))
        opt.step()
        assert np.isclose(o.grad_norm([g]), norm, rtol=1e-14)
        p, m, v = o.adamw(p, m, v, g, 0.01, step, 0.8, 0.99, 1e-6, 0.1, o.clip_factor(norm, 3.0))
        assert np.allclose(t.detach().numpy(), p, rtol=1e-12, atol=1e-14)
