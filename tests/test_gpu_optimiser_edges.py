"""Tensor lists where a scalar, a gradient or the size is out of the ordinary.  (Bounds of a step: test_gpu_optimiser.py.)"""
import pytest
import torch

from oracle import optimiser as o
from test_gpu_optimiser import check_step, grads_of, norm_close, state_of
from util_gpu import to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    import paper_2501_14183_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(vd):
    return vd.Context(0)


def whole_list(vd, ctx, sizes=(5000, 7)):
    """A list with everything AdamW takes, its state, and a copy of that."""
    state = [[torch.rand(n, device="cuda") + 0.5 for n in sizes] for _ in range(4)]
    tensors = vd.TensorList(ctx, state[0], params=state[1], exp_avg=state[2], exp_avg_sq=state[3])
    return tensors, state, [[t.clone() for t in k] for k in state]


def unchanged(state, kept):
    return all(torch.equal(a, b) for x, y in zip(state, kept) for a, b in zip(x, y))


@pytest.mark.parametrize("bad", [dict(eps=1e-46), dict(eps=1e-300), dict(eps=1e39), dict(lr=1e39), dict(lr=1e38, step=1)],
                         ids=lambda b: "-".join("%s=%g" % kv for kv in b.items()))
def test_scalars_that_single_precision_does_not_hold_are_refused(vd, ctx, bad):
    """eps that rounds to zero would divide zero moments by zero; a rate (or one over 1 - beta1^step) past the range is infinite."""
    tensors, state, kept = whole_list(vd, ctx)
    for k in (2, 3):
        for a, b in zip(state[k], kept[k]):
            a.zero_()
            b.zero_()
    with pytest.raises(vd.VarDropError) as e:
        vd.vardrop_adamw(ctx, tensors, **{**dict(lr=0.1, step=3), **bad})
    assert e.value.code == -1 and unchanged(state, kept)


def test_the_smallest_eps_is_taken(vd, ctx):
    tensors, state, _ = whole_list(vd, ctx)
    for t in state[0] + state[2] + state[3]:
        t.zero_()
    kept = [t.clone() for t in state[1]]
    vd.vardrop_adamw(ctx, tensors, 0.1, 1, eps=1.5e-45)
    assert all(torch.equal(a, b) for a, b in zip(state[1], kept))


@pytest.mark.parametrize("rate,step", [(float("nan"), 3), (float("inf"), 3), (-0.1, 3), (0.1, -1), (0.1, -5), (1e38, 0)])
def test_a_device_rate_or_counter_out_of_range_skips_the_step(vd, ctx, rate, step):
    """What the call with host scalars refuses, the one that reads them on the device cannot: it writes nothing and says so."""
    tensors, state, kept = whole_list(vd, ctx, (5000, 7, 4096 * 40))
    rate_dev, status = torch.full((1,), rate, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    step_dev = torch.full((1,), step, dtype=torch.int64, device="cuda")
    vd.vardrop_adamw_dev(ctx, tensors, rate_dev, step_dev, status=status)
    assert int(status) == 1 and int(step_dev) == step and unchanged(state, kept)
    # the list and its counters work again
    rate_dev.fill_(0.1)
    step_dev.fill_(2)
    status.zero_()
    vd.vardrop_adamw_dev(ctx, tensors, rate_dev, step_dev, status=status)
    assert int(status) == 0 and int(step_dev) == 3
    again, state2, _ = whole_list(vd, ctx, (5000, 7, 4096 * 40))
    for a, b in zip(state2, kept):
        for x, y in zip(a, b):
            x.copy_(y)
    vd.vardrop_adamw(ctx, again, float(rate_dev), 3)
    assert unchanged(state, state2)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("to", [torch.float32, torch.bfloat16])
def test_clipped_gradients_are_never_those_of_an_earlier_step(vd, ctx, value, to):
    """With a norm that is not finite the clip tensors get what the formula gives (g times max_norm / norm: zero or not a number)."""
    host, grads = grads_of([4097, 30], 7)
    out = [torch.empty(g.numel(), dtype=to, device="cuda") for g in grads]
    tensors = vd.TensorList(ctx, grads, clipped=out)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    vd.vardrop_clip_grads(ctx, tensors, vd.vardrop_grad_norm(ctx, tensors), 0.5, status=status)
    assert int(status) == 0 and all(bool(c.any()) for c in out)
    grads[0][4096] = value
    norm = vd.vardrop_grad_norm(ctx, tensors)
    vd.vardrop_clip_grads(ctx, tensors, norm, 0.5, status=status)
    assert int(status) == 1
    for g, c in zip(grads, out):
        want = (g * (0.5 / (norm + 1e-6))).to(to)
        assert torch.equal(c.nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("low", [False, True])
def test_a_large_model_steps_on_the_device(vd, ctx, low):
    """9.6 million weights in 2347 chunks: weights past the caches, counters shared by more than 32 workgroups, norms of workgroups with
    several chunks; three steps in a row, each against the oracle."""
    sizes = [4500001, 3, 3000017, 900003, 777777, 409600]
    host, grads = grads_of(sizes, 11, ("bf16", "fp32"))
    dev = [[to_dev(a) for a in k] for k in state_of(sizes, 12, True)]
    weights = [torch.empty(n, dtype=torch.bfloat16, device="cuda") if low or i % 2 else None for i, n in enumerate(sizes)]
    decay = [0.1 * (i % 2) for i in range(len(sizes))]
    tensors = vd.TensorList(ctx, grads, params=dev[0], exp_avg=dev[1], exp_avg_sq=dev[2], weights=weights, decay=decay)
    assert tensors.struct.chunks > 2048 and tensors.struct.numel > 6000000
    step, rate = torch.full((1,), 40, dtype=torch.int64, device="cuda"), torch.full((1,), 0.01, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lr = float(rate)
    for k in range(41, 44):
        before = [[t.cpu().numpy() for t in a] for a in dev]
        norm = vd.vardrop_grad_norm(ctx, tensors)
        norm_close(norm, o.grad_norm(host))
        vd.vardrop_adamw_dev(ctx, tensors, rate, step, beta1=0.9, beta2=0.99, eps=1e-7, norm=norm, max_norm=0.3, status=status)
        assert int(step) == k and int(status) == 0
        check_step(host, before, dev, lr, k, decay, o.clip_factor(o.grad_norm(host), 0.3), 0.9, 0.99, 1e-7, weights)
        for i, g in enumerate(grads):
            g.mul_(-0.5)
            host[i] = -0.5 * host[i]
