"""Products in 8-bit integers (vardrop_quantize_rows, vardrop_quantize_weight, vardrop_linear_i8) against the oracle.

Codes and scales are equal.  The integer sum is exact; its conversion to fp32, two scales, the bias: 6 u of the magnitudes; GELU as in
util_ffn.py; a result in bf16 is rounded once more, by at most 2^-8."""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import feedforward as o
from util_ffn import BF, U, act_error
from util_gpu import to_dev, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    import paper_2501_14183_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(vd):
    return vd.Context(0)


def make(T, K, N, dtype, bias=True):
    rng = np.random.default_rng([0x18, T, K, N])
    x = wl.quantise(rng.standard_normal((T, K)) * np.exp(rng.uniform(-2, 2, K)) * np.exp(rng.uniform(-5, 5, (T, 1))), dtype)
    W = wl.quantise(rng.standard_normal((K, N)) / K ** 0.5 * np.exp(rng.uniform(-3, 3, N)), dtype)
    return x, W, wl.quantise(rng.standard_normal(N), dtype) if bias else None


def check_codes(codes, scale, want, K):
    q, s = want
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)
    host = codes.cpu().numpy()
    assert np.array_equal(host[:, :K], q) and not host[:, K:].any()


def bound(x, W, b, act, dtype):
    v = o.linear_i8(x, W, b, "none")
    want = o.linear_i8(x, W, b, act)
    e = 6 * U * (np.abs(v) + 2 * (0 if b is None else np.abs(b)))
    e = e if act == "none" else act_error(v, e, dtype, act)
    return want, e if dtype == "fp32" else e + BF * (np.abs(want) + e)


SIZES = [(7, 512, 100), (8, 2048, 33), (9, 1024, 130), (64, 1025, 128), (129, 600, 200), (862, 512, 720), (1, 1, 1), (1, 512, 512), (2, 3, 5), (5, 97, 33), (1, 128, 64), (3, 129, 127), (16, 64, 128), (17, 200, 129), (63, 96, 321), (64, 128, 8), (65, 257, 130),
         (130, 1000, 72), (200, 2048, 40), (300, 2050, 24), (257, 31, 700)]


@pytest.mark.parametrize("dtype,act", [("fp32", "none"), ("bf16", "gelu"), ("fp32", "gelu"), ("bf16", "relu")])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_equal_codes_and_near_products(vd, ctx, T, K, N, dtype, act):
    x, W, b = make(T, K, N, dtype)
    dt = torch_dtype(dtype)
    tx, tW, tb = to_dev(x, dt), to_dev(W, dt), to_dev(b, dt)
    codes, scale = vd.vardrop_quantize_weight(ctx, tW)
    check_codes(codes, scale, o.integers(np.ascontiguousarray(W.T)), K)
    q, s = vd.vardrop_quantize_rows(ctx, tx)
    check_codes(q, s, o.integers(x), K)
    kind = {"none": vd.ACT_NONE, "relu": vd.ACT_RELU, "gelu": vd.ACT_GELU}[act]
    room = torch.full((T * N + 64,), 7.0, dtype=dt, device="cuda")
    y = vd.vardrop_linear_i8(ctx, tx, codes, scale, tb, act=kind, out=room[:T * N].view(T, N))
    want, e = bound(x, W, b, act, dtype)
    off = np.abs(y.double().cpu().numpy() - want)
    assert (off <= e).all(), float((off / np.maximum(e, 1e-300)).max())
    assert bool((room[T * N:] == 7.0).all())
    again = vd.vardrop_linear_i8(ctx, (q, s), codes, scale, tb, act=kind, dtype=dt)
    assert torch.equal(again, y)


@pytest.mark.parametrize("T,K,N", [(9000, 64, 1000), (70000, 40, 65)])
def test_many_tokens(vd, ctx, T, K, N):
    x, W, b = make(T, K, N, "bf16", bias=False)
    tx = to_dev(x, torch.bfloat16)
    codes, scale = vd.vardrop_quantize_weight(ctx, to_dev(W, torch.bfloat16))
    y = vd.vardrop_linear_i8(ctx, tx, codes, scale)
    want, e = bound(x, W, None, "none", "bf16")
    assert (np.abs(y.double().cpu().numpy() - want) <= e).all()


def test_the_largest_sum(vd, ctx):
    """65 536 products of 127 and 127: the sum does not fit 30 bits."""
    K = 65536
    x = torch.full((2, K), 3.0, device="cuda")
    x[1] = -3.0
    codes, scale = vd.vardrop_quantize_weight(ctx, torch.full((K, 3), 0.5, device="cuda"))
    y = vd.vardrop_linear_i8(ctx, x, codes, scale)
    assert np.allclose(y.double().cpu().numpy(), [[1.5 * K] * 3, [-1.5 * K] * 3], rtol=8 * U)


def test_rows_that_have_no_scale(vd, ctx):
    """Zeros and numbers too small for one count as zeros; an infinity or NaN spoils its row, and its column, alone."""
    x = torch.randn(6, 130, device="cuda")
    x[1], x[2], x[3, 7], x[4, 129] = 0.0, 1e-36, float("inf"), float("nan")
    W = torch.randn(130, 20, device="cuda")
    W[:, 3], W[5, 11] = 0.0, float("-inf")
    b = torch.randn(20, device="cuda")
    y = vd.vardrop_linear_i8(ctx, x, *vd.vardrop_quantize_weight(ctx, W), b)
    ok = torch.ones(6, 20, dtype=torch.bool, device="cuda")
    ok[3:5], ok[:, 11] = False, False
    assert torch.equal(torch.isfinite(y), ok) and bool(torch.isnan(y[~ok]).all())
    some = torch.tensor([c for c in range(20) if c != 11], device="cuda")
    assert torch.equal(y[1][some], b[some]) and torch.equal(y[2][some], b[some]) and torch.equal(y[:, 3][ok[:, 3]], b[3].expand(4))


def test_types_and_shapes_mix(vd, ctx):
    """A batch of any rank, x and y of different types, rows and results that begin at any element."""
    x, W, b = make(42, 96, 50, "bf16")
    codes, scale = vd.vardrop_quantize_weight(ctx, to_dev(W).float())
    check_codes(codes, scale, o.integers(np.ascontiguousarray(W.T)), 96)
    room = torch.zeros(42 * 96 + 3, dtype=torch.bfloat16, device="cuda")
    t = room[3:].view(2, 3, 7, 96)
    t.copy_(to_dev(x).view(2, 3, 7, 96))
    y = vd.vardrop_linear_i8(ctx, t, codes, scale, to_dev(b).float())
    assert y.shape == (2, 3, 7, 50) and y.dtype is torch.float32
    want, e = bound(x, W, b, "none", "fp32")
    assert (np.abs(y.double().cpu().numpy().reshape(42, 50) - want) <= e).all()
    out = torch.zeros(42 * 50 + 1, dtype=torch.bfloat16, device="cuda")
    low = vd.vardrop_linear_i8(ctx, t, codes, scale, to_dev(b, torch.bfloat16), out=out[1:].view(42, 50))
    assert torch.equal(low, y.bfloat16().view(42, 50)) and float(out[0]) == 0.0


def test_a_block_that_answers(vd, ctx):
    """Two products with GELU between them, as a served feed-forward block runs them, recorded and replayed."""
    rng = np.random.default_rng(4)
    d, f = 64, 160
    W = [wl.quantise(rng.standard_normal(s) / s[0] ** 0.5, "bf16") for s in ((d, f), (f, d))]
    up, down = (vd.vardrop_quantize_weight(ctx, to_dev(w, torch.bfloat16)) for w in W)
    for T in (1, 90):
        x = to_dev(wl.quantise(rng.standard_normal((T, d)), "bf16"), torch.bfloat16)
        a, y = torch.zeros(T, f, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
        ws = torch.zeros(max(vd.vardrop_linear_i8_workspace_bytes(T, k, n) for k, n in ((d, f), (f, d))), dtype=torch.uint8, device="cuda")

        def answer():
            vd.vardrop_linear_i8(ctx, x, *up, act=vd.ACT_GELU, ws=ws, out=a)
            vd.vardrop_linear_i8(ctx, a, *down, ws=ws, out=y)

        answer()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            answer()
        for _ in range(3):
            x.copy_(to_dev(wl.quantise(rng.standard_normal((T, d)), "bf16")))
            graph.replay()
            got = y.clone()
            answer()
            torch.cuda.synchronize()
            assert torch.equal(got, y)
            full = o.activation("gelu", x.double().cpu().numpy() @ W[0]) @ W[1]
            # codes are off by half a step of 1/127 of a row's largest: 0.4 % of it, in a sum of independent errors
            assert np.sqrt(((y.double().cpu().numpy() - full) ** 2).sum()) <= 0.04 * np.sqrt((full ** 2).sum())


def test_refusals(vd, ctx):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")
    x, W = z(4, 96), z(96, 50)
    codes, scale = vd.vardrop_quantize_weight(ctx, W)
    ws = z(vd.vardrop_linear_i8_workspace_bytes(4, 96, 50) + 256, dt=torch.uint8)
    q, s = vd.vardrop_quantize_rows(ctx, x)
    calls = [
        lambda: vd.vardrop_quantize_weight(ctx, W.half()), lambda: vd.vardrop_quantize_weight(ctx, W.t()), lambda: vd.vardrop_quantize_weight(ctx, W.cpu()),
        lambda: vd.vardrop_quantize_rows(ctx, x.half()), lambda: vd.vardrop_quantize_rows(ctx, z(1, 70000)), lambda: vd.vardrop_quantize_rows(ctx, z(4, 0)),
        lambda: vd.vardrop_linear_i8(ctx, z(4, 300), codes, scale), lambda: vd.vardrop_linear_i8(ctx, x, codes[:49], scale),
        lambda: vd.vardrop_linear_i8(ctx, x, codes, scale.half()), lambda: vd.vardrop_linear_i8(ctx, x, codes, scale, bias=z(49)),
        lambda: vd.vardrop_linear_i8(ctx, x, codes, scale, act=3), lambda: vd.vardrop_linear_i8(ctx, x, codes, scale, out=z(4, 49)),
        lambda: vd.vardrop_linear_i8(ctx, x, codes, scale, ws=ws[:256]), lambda: vd.vardrop_linear_i8(ctx, x, codes, scale, ws=ws[1:]),
        lambda: vd.vardrop_linear_i8(ctx, (q, s[:3]), codes, scale), lambda: vd.vardrop_linear_i8(ctx, (q[:, :96], s), codes, scale),
        lambda: vd.vardrop_linear_i8(ctx, x, codes, scale, stream=0), lambda: vd.vardrop_linear_i8(ctx, x, codes, scale, dtype=torch.float16),
        lambda: vd.vardrop_linear_i8(ctx, x.cpu(), codes, scale),
    ]
    for k, call in enumerate(calls):
        with pytest.raises((TypeError, ZeroDivisionError, vd.VarDropError)):
            call()
            pytest.fail("call %d was taken" % k)
    assert vd.vardrop_linear_i8(ctx, z(0, 96), codes, scale).shape == (0, 50)
