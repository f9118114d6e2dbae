"""Activations in 8 bits (vardrop_pack8 / vardrop_unpack8) against the fp64 oracle: equal, byte for byte."""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import feedforward as o
from util_gpu import to_dev, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    import paper_2501_14183_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(vd):
    return vd.Context(0)


def bytes_of(saved, rows, d):
    """Codes and exponent bytes of a checkpoint."""
    host = saved.cpu().numpy()
    nb, at = -(-d // 32), -(-rows * d // 256) * 256
    return host[:rows * d].view(np.int8).reshape(rows, d), host[at:at + rows * nb].reshape(rows, nb)


def check(vd, ctx, x, dtype, want_codes, want_exps):
    t = to_dev(x, torch_dtype(dtype))
    B, n, d = t.shape
    size = vd.vardrop_pack8_bytes(B, n, d)
    buf = torch.full((size + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    saved = vd.vardrop_pack8(ctx, t, out=buf[:size])
    codes, exps = bytes_of(saved, B * n, d)
    assert np.array_equal(exps, want_exps)
    good = np.repeat(want_exps != 255, 32, axis=1)[:, :d]
    assert np.array_equal(codes[good], want_codes[good])
    assert bool((buf[size:] == 0xAB).all())
    want = torch.from_numpy(o.unpack8(want_codes, want_exps).reshape(x.shape))
    for other in ("fp32", "bf16"):
        room = torch.full((B * n * d + 64,), 7.0, dtype=torch_dtype(other), device="cuda")
        back = vd.vardrop_unpack8(ctx, saved, room[:B * n * d].view(B, n, d))
        assert torch.equal(torch.nan_to_num(back.double().cpu(), nan=-1e300), torch.nan_to_num(want, nan=-1e300))
        assert bool((room[B * n * d:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 1, 32), (1, 3, 31), (2, 1, 33), (3, 5, 64), (1, 7, 97), (4, 10, 64), (2, 33, 320), (3, 41, 321),
                                   (1, 9, 1504), (2, 700, 96)])
def test_equal_to_the_oracle(vd, ctx, shape, dtype):
    rng = np.random.default_rng([8, *shape])
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-6, 6, shape[-1]))
    x.reshape(-1)[rng.integers(x.size, size=1 + x.size // 50)] = 0.0
    x = wl.quantise(x, dtype)
    check(vd, ctx, x, dtype, *o.pack8(x.reshape(-1, shape[-1])))


@pytest.mark.parametrize("d", [32, 70])
def test_the_ends_of_the_range(vd, ctx, d):
    """Zeros, numbers too small for a step, the largest, ties, infinities and NaN."""
    x = np.zeros((1, 12, d), dtype=np.float32)
    x[0, 1] = 2.0 ** -140
    x[0, 2, ::2] = 2.0 ** -126
    x[0, 3] = np.linspace(-3.4e38, 3.4e38, d)
    x[0, 4] = np.arange(d) - 0.5
    x[0, 5] = 127.5 * 2.0 ** -20
    x[0, 6, 0] = np.inf
    x[0, 7, d - 1] = np.nan
    x[0, 8, 3] = -np.inf
    x[0, 9] = 2.0 ** -119 * 1.9921875
    x[0, 10] = -0.0
    x[0, 11] = np.float32(1.9921874) * np.float32(2.0) ** 5
    check(vd, ctx, x, "fp32", *o.pack8(x[0]))


def test_rows_need_element_alignment_only(vd, ctx):
    rng = np.random.default_rng(9)
    for d in (32, 64, 50):
        x = wl.quantise(rng.standard_normal((2, 5, d)), "bf16")
        room = torch.zeros(x.size + 1, dtype=torch.bfloat16, device="cuda")
        t = room[1:].view(2, 5, d)
        t.copy_(to_dev(x))
        saved = vd.vardrop_pack8(ctx, t)
        codes, exps = bytes_of(saved, 10, d)
        want_codes, want_exps = o.pack8(x.reshape(10, d))
        assert np.array_equal(codes, want_codes) and np.array_equal(exps, want_exps)
        out = torch.zeros_like(room)
        back = vd.vardrop_unpack8(ctx, saved, out[1:].view(2, 5, d))
        assert np.array_equal(back.double().cpu().numpy().reshape(10, d), o.unpack8(want_codes, want_exps)) and float(out[0]) == 0.0


@pytest.mark.parametrize("d", [64, 70])
def test_a_count_on_the_device(vd, ctx, d):
    B, n_max = 3, 20
    rng = np.random.default_rng(10)
    for n in (0, 1, 7, 20, 21, -1):
        live = max(0, min(n, n_max)) if 0 <= n <= n_max else 0
        x = wl.quantise(rng.standard_normal((B, n_max, d)), "bf16")
        t = to_dev(x, torch.bfloat16)
        n_dev, status = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        saved = torch.full((vd.vardrop_pack8_bytes(B, n_max, d),), 0x55, dtype=torch.uint8, device="cuda")
        vd.vardrop_pack8(ctx, t, out=saved, n_dev=n_dev, status=status)
        assert int(status) == (0 if 0 <= n <= n_max else 1)
        out = torch.full((B, n_max, d), 9.0, dtype=torch.float32, device="cuda")
        status.zero_()
        vd.vardrop_unpack8(ctx, saved, out, n_dev=n_dev, status=status)
        assert int(status) == (0 if 0 <= n <= n_max else 1)
        rows = B * live
        want = o.through_8_bits(x.reshape(-1, d)[:rows]) if rows else np.zeros((0, d))
        assert np.array_equal(out.double().cpu().numpy().reshape(-1, d)[:rows], want)
        assert bool((out.reshape(-1, d)[rows:] == 9.0).all()) and bool((saved[rows * d:B * n_max * d] == 0x55).all())


def test_refusals(vd, ctx):
    x = torch.zeros(2, 3, 64, device="cuda")
    saved = vd.vardrop_pack8(ctx, x)
    bad = torch.zeros(vd.vardrop_pack8_bytes(2, 3, 64) + 256, dtype=torch.uint8, device="cuda")
    for call in (lambda: vd.vardrop_pack8(ctx, x.half()), lambda: vd.vardrop_pack8(ctx, x.transpose(0, 1)), lambda: vd.vardrop_pack8(ctx, x, out=bad[1:]),
                 lambda: vd.vardrop_pack8(ctx, x, out=bad[:100]), lambda: vd.vardrop_unpack8(ctx, saved, x.cpu()),
                 lambda: vd.vardrop_unpack8(ctx, saved[:256], x), lambda: vd.vardrop_pack8(ctx, x, stream=0),
                 lambda: vd.vardrop_pack8(ctx, x, n_dev=torch.zeros(1, device="cuda"))):
        with pytest.raises((TypeError, vd.VarDropError)):
            call()
    empty = torch.zeros(0, 3, 64, device="cuda")
    assert vd.vardrop_unpack8(ctx, vd.vardrop_pack8(ctx, empty), empty).numel() == 0
