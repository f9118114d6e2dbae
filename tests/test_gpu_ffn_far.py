"""Feed-forward block, 8-bit checkpoints and 8-bit products whose buffers are longer than 32-bit offsets reach, and the longest rows."""
import pytest
import torch

import util_ffn_tiles as u

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def vd():
    import paper_2501_14183_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(vd):
    return vd.Context(0)


@pytest.fixture(autouse=True)
def free():
    yield
    torch.cuda.empty_cache()


def random(dt, *shape, seed=0):
    return torch.empty(*shape, dtype=dt, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(seed))


@pytest.mark.parametrize("n,d", [(3, 1 << 20), (3, (1 << 20) - 1), (2, 1 << 16)])
def test_checkpoints_of_the_longest_rows(vd, ctx, n, d):
    x = random(F32, n, d, seed=n)
    saved = vd.vardrop_pack8(ctx, x.view(1, n, d))
    codes, exps, values = u.pack(x)
    at = -(-n * d // 256) * 256
    assert torch.equal(saved[:n * d].view(torch.int8).view(n, d), codes) and torch.equal(saved[at:at + exps.numel()].view(exps.shape), exps)
    assert torch.equal(vd.vardrop_unpack8(ctx, saved, torch.empty(1, n, d, device="cuda"))[0].to(u.F64), values)


@pytest.mark.parametrize("n,d", [(4_500_001, 512), (6_900_001, 321)])
def test_checkpoints_of_more_than_2_31_elements(vd, ctx, n, d):
    """The last rows are those of a call of their own."""
    assert n * d > 1 << 31
    x, last = random(BF16, n, d, seed=1), 1000
    saved = vd.vardrop_pack8(ctx, x.view(1, n, d))
    own = vd.vardrop_pack8(ctx, x[-last:].contiguous().view(1, last, d))
    assert torch.equal(saved[(n - last) * d:n * d], own[:last * d])
    nb, at, at_own = -(-d // 32), -(-n * d // 256) * 256, -(-last * d // 256) * 256
    assert torch.equal(saved[at + (n - last) * nb:at + n * nb], own[at_own:at_own + last * nb])
    back = vd.vardrop_unpack8(ctx, saved, torch.empty(1, n, d, dtype=BF16, device="cuda"))[0]
    assert torch.equal(back[-last:].to(u.F64), u.pack(x[-last:])[2])


@pytest.mark.parametrize("dt", [BF16, F32])
def test_products_of_more_rows_than_4_gb_hold(vd, ctx, dt):
    """Codes of 5 GB, results past 2^31 bytes: the last rows are those of a call of their own."""
    rows, K, N, last = 40_000_003, 24, 17, 700
    x, W = random(dt, rows, K, seed=2), random(dt, K, N, seed=3)
    weight = vd.vardrop_quantize_weight(ctx, W)
    y = vd.vardrop_linear_i8(ctx, x, *weight)
    assert torch.equal(y[-last:], vd.vardrop_linear_i8(ctx, x[-last:].contiguous(), *weight))
    q, s = vd.vardrop_quantize_rows(ctx, x)
    own = vd.vardrop_quantize_rows(ctx, x[-last:].contiguous())
    assert torch.equal(q[-last:], own[0]) and torch.equal(s[-last:], own[1])
    del y
    assert torch.equal(vd.vardrop_linear_i8(ctx, (q, s), *weight, dtype=dt)[-last:], vd.vardrop_linear_i8(ctx, own, *weight, dtype=dt))


@pytest.mark.parametrize("rows", [1, 3, 70, 300])
def test_products_of_more_channels_than_4_gb_hold(vd, ctx, rows):
    """Codes of a weight of 5 GB."""
    K, N, last = 24, 40_000_003, 131
    x, W = random(BF16, rows, K, seed=4), random(BF16, K, N, seed=5)
    codes, scale = vd.vardrop_quantize_weight(ctx, W)
    own = vd.vardrop_quantize_weight(ctx, W[:, -last:].contiguous())
    assert torch.equal(codes[-last:], own[0]) and torch.equal(scale[-last:], own[1])
    y = vd.vardrop_linear_i8(ctx, x, codes, scale)
    assert torch.equal(y[:, -last:], vd.vardrop_linear_i8(ctx, x, *own))


@pytest.mark.parametrize("T,d,f", [(5, 46336, 46336), (300, 65536, 32704)])
def test_weights_of_almost_2_31_elements(vd, ctx, T, d, f):
    """Whole numbers, as in util_ffn_tiles.py, of which some columns and rows are compared."""
    assert (1 << 31) - d * f < 1 << 23
    g = torch.Generator("cuda").manual_seed(6)
    p = (150 * 9 / 4 / d) ** 0.5

    def signs(*shape):
        """-1, 0, 1, made in the type of the block."""
        t = torch.empty(*shape, dtype=BF16, device="cuda").uniform_(-1, 1, generator=g)
        return t.abs().lt(p * 2 / 3).to(BF16).mul_(t.sign())

    x, W1, W2, dy = signs(T, d), signs(d, f), signs(f, d), signs(T, d)
    b1, b2 = torch.randint(-8, 9, (f,), generator=g, device="cuda").to(BF16), torch.randint(-8, 9, (d,), generator=g, device="cuda").to(BF16)
    y, saved = vd.vardrop_ffn_fwd(ctx, x.view(1, T, d), W1, W2, b1, b2, act=vd.ACT_RELU)
    dx, dW1, dW2, db1, db2 = vd.vardrop_ffn_bwd(ctx, dy.view(1, T, d), W1, W2, saved, act=vd.ACT_RELU, bias_grads=True)

    def product(A, B):
        """A @ B of whole numbers, in pieces of the summed axis."""
        return sum(A[:, k:k + 4096].to(u.F64) @ B[k:k + 4096].to(u.F64) for k in range(0, A.shape[1], 4096))

    h = product(x, W1) + b1.to(u.F64)
    da = torch.cat([product(dy, W2[k:k + 4096].t()) for k in range(0, f, 4096)], 1)
    assert float(h.abs().max()) <= 127 and float(da.abs().max()) <= 256
    a, dh = h.clamp(min=0), da * (h > 0)
    same = lambda got, want: torch.equal(got, want.to(F32).to(got.dtype))
    assert same(y[0], product(a, W2) + b2.to(u.F64))
    assert same(dx[0], torch.cat([product(dh, W1[k:k + 4096].t()) for k in range(0, d, 4096)], 1))
    assert same(db1, dh.sum(0)) and same(db2, dy.to(u.F64).sum(0))
    for k in (0, d // 2, d - 64):
        assert same(dW1[k:k + 64], x[:, k:k + 64].t().to(u.F64) @ dh)
    for k in (0, f // 2, f - 64):
        assert same(dW2[k:k + 64], a[:, k:k + 64].t() @ dy.to(u.F64))


@pytest.mark.parametrize("B,n,d,f", [(1, 300, 64, 192), (1, 9001, 448, 1600)])
def test_the_first_call_may_be_a_captured_one(vd, B, n, d, f):
    """A graph recorded by a context that has made no call, then replayed over other inputs beside eager calls."""
    ctx = vd.Context(0)
    t = {k: v.to(BF16) for k, v in u.dense(B * n, d, f).items()}
    x, dy = t["x"].view(B, n, d), t["dy"].view(B, n, d)
    room = lambda size: torch.zeros(size, dtype=torch.uint8, device="cuda")
    y, saved, ws = torch.zeros_like(x), room(vd.vardrop_ffn_saved_bytes(B, n, d, f)), room(vd.vardrop_ffn_workspace_bytes(B, n, d, f, BF16))
    grads = (torch.zeros_like(x), *[torch.zeros(s, device="cuda") for s in ((d, f), (f, d), (f,), (d,))])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vd.vardrop_ffn_fwd(ctx, x, t["W1"], t["W2"], t["b1"], t["b2"], saved=saved, ws=ws, out=y)
        vd.vardrop_ffn_bwd(ctx, dy, t["W1"], t["W2"], saved, ws=ws, out=grads)
    for k in range(3):
        x.copy_(random(BF16, B, n, d, seed=20 + k))
        graph.replay()
        want, kept = vd.vardrop_ffn_fwd(ctx, x, t["W1"], t["W2"], t["b1"], t["b2"])
        wanted = vd.vardrop_ffn_bwd(ctx, dy, t["W1"], t["W2"], kept, bias_grads=True)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(grads, wanted))
