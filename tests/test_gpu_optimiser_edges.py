"""Tensor lists where a scalar or a gradient is out of the ordinary."""
import pytest
import torch

from test_gpu_optimiser import grads_of

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
