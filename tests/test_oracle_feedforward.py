"""The oracle of the feed-forward block: its checkpoints' format, and its gradients against differences."""
import numpy as np
import pytest

from oracle import feedforward as o


def test_a_block_is_whole_numbers_of_its_step():
    x = np.zeros((1, 40))
    x[0, :4] = (1.0, -0.5, 0.3, 127.0)
    x[0, 39] = 2.0 ** -130
    codes, exps = o.pack8(x)
    assert list(codes[0, :4]) == [1, 0, 0, 127] and exps[0, 0] == 127          # -0.5 is a tie and goes to the even one
    assert exps[0, 1] == 1 and codes[0, 39] == 0
    assert list(o.unpack8(codes, exps)[0, :4]) == [1.0, 0.0, 0.0, 127.0]


@pytest.mark.parametrize("most,step", [(127.0, 1.0), (127.49, 1.0), (127.5, 2.0), (128.0, 2.0), (64.0, 1.0), (63.7, 0.5), (63.75, 1.0)])
def test_the_step_is_the_smallest_that_holds_the_largest(most, step):
    codes, exps = o.pack8(np.full((1, 1), most))
    assert 2.0 ** (int(exps[0, 0]) - 127) == step
    assert abs(float(o.unpack8(codes, exps)[0, 0]) - most) <= step / 2


def test_values_are_within_half_a_step_and_bf16():
    x = np.random.default_rng(1).standard_normal((50, 77)) * np.exp(np.random.default_rng(2).uniform(-20, 20, (50, 1)))
    back = o.through_8_bits(x)
    for b in range(0, 77, 32):
        most = np.abs(x[:, b:b + 32]).max(1, keepdims=True)
        assert (np.abs(back - x)[:, b:b + 32] <= most * 2.0 ** -7 * 1.005).all()
    as_bits = back.astype(np.float32).view(np.uint32)
    assert (as_bits & 0xffff == 0).all() and (back.astype(np.float32) == back).all()
    assert (o.through_8_bits(back) == back).all()


def test_what_is_not_finite_spoils_its_block_alone():
    x = np.ones((2, 96))
    x[0, 40], x[1, 95] = np.inf, np.nan
    back = o.through_8_bits(x)
    assert np.isnan(back[0, 32:64]).all() and np.isnan(back[1, 64:]).all() and np.isfinite(back).sum() == 128
    assert float(o.through_8_bits(np.full((1, 1), 3.4e38))[0, 0]) == 127 * 2.0 ** 121


@pytest.mark.parametrize("act", ["relu", "gelu"])
def test_gradients_are_differences(act):
    rng = np.random.default_rng(3)
    T, d, f = 5, 6, 7
    p = dict(x=rng.standard_normal((T, d)), W1=rng.standard_normal((d, f)), b1=rng.standard_normal(f), W2=rng.standard_normal((f, d)),
             b2=rng.standard_normal(d))
    dy = rng.standard_normal((T, d))

    def loss(**kw):
        return float((o.forward(**{**p, **kw}, act=act)[0] * dy).sum())

    h = o.forward(**p, act=act)[1]
    got = o.backward(dy, p["x"], h, p["W1"], p["W2"], act)
    for name in p:
        want = np.zeros_like(p[name])
        for at in np.ndindex(*want.shape):
            lo, hi = p[name].copy(), p[name].copy()
            lo[at] -= 1e-6
            hi[at] += 1e-6
            want[at] = (loss(**{name: hi}) - loss(**{name: lo})) / 2e-6
        assert np.allclose(got["d" + name], want, rtol=1e-6, atol=1e-6)


def test_integers_are_exact_where_the_scale_allows():
    x = np.array([[127.0, -3.0, 0.5], [0.0, 0.0, 0.0], [1e-38, 0.0, 0.0], [np.inf, 1.0, 0.0]], dtype=np.float32)
    codes, scale = o.integers(x)
    assert list(codes[0]) == [127, -3, 0] and scale[0] == 1.0
    assert scale[1] == 0 and scale[2] == 0 and np.isnan(scale[3]) and not codes[1:].any()
    W = np.eye(3, dtype=np.float32) * 127
    assert np.allclose(o.linear_i8(x[:1], W, np.ones(3), "none"), [[127 * 127 + 1, -3 * 127 + 1, 1.0]])
