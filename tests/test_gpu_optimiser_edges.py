"""Tensor lists where a scalar or a gradient is out of the ordinary."""
import pytest
import torch

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
