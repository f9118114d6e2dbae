"""The feed-forward block in every tile that its sizes select, and the 8-bit products in theirs, against definitions in 64 bits; inputs and bounds in
util_ffn_tiles.py."""
import pytest
import torch

import util_ffn_tiles as u
from util_ffn import BF, U

pytestmark = pytest.mark.gpu
NAMES = ("dx", "dW1", "dW2", "db1", "db2")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def vd():
    import paper_2501_14183_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(vd):
    return vd.Context(0)


def rooms(*shapes, dtype):
    """Tensors with a margin of sevens behind each, and the margins."""
    made = [torch.full((torch.Size(s).numel() + 64,), 7.0, dtype=dtype, device="cuda") for s in shapes]
    return [r[:-64].view(s) for r, s in zip(made, shapes)], [r[-64:] for r in made]


def same(name, got, want):
    """Equal to the definition after one rounding."""
    want = want.to(F32).to(got.dtype).reshape(got.shape)
    wrong = got != want
    assert not bool(wrong.any()), "%s: %d of %d differ, first at %s" % (name, int(wrong.sum()), wrong.numel(), wrong.nonzero()[0].tolist())


def whole_block(vd, ctx, B, n, d, f, dt, gt, n_max=None):
    """Whole numbers through both ways, equal to the definition; n_max: a buffer for so many tokens, the count on the device."""
    t = u.whole_numbers(B, n, d, f)
    w = u.wide(t)
    y64, h64 = u.forward(w, "relu")
    assert float(h64.abs().max()) <= 127 and float((w["dy"] @ w["W2"].t()).abs().max()) <= 256
    want = u.backward(w, w["x"], h64, "relu")
    assert all(float(v.abs().max()) < 2 ** 24 for v in (y64, *want.values()))
    del h64
    g, kw, most = {k: v.to(dt) for k, v in t.items()}, {}, n if n_max is None else n_max
    if n_max is not None:
        kw = dict(n_dev=torch.tensor([n], dtype=torch.int32, device="cuda"), status=torch.zeros(1, dtype=torch.int32, device="cuda"))
        for k in ("x", "dy"):
            room = torch.full((B * n_max, d), float("nan"), dtype=dt, device="cuda")
            room[:B * n] = g[k]
            g[k] = room
    x, dy = (g[k].view(B, most, d) for k in ("x", "dy"))
    (y, dx), ends = rooms((B, most, d), (B, most, d), dtype=dt)
    saved = torch.full((vd.vardrop_ffn_saved_bytes(B, most, d, f),), 0xFF, dtype=torch.uint8, device="cuda")
    ws = torch.full((vd.vardrop_ffn_workspace_bytes(B, most, d, f, dt),), 0xFF, dtype=torch.uint8, device="cuda")
    vd.vardrop_ffn_fwd(ctx, x, g["W1"], g["W2"], g["b1"], g["b2"], act=vd.ACT_RELU, saved=saved, ws=ws, out=y, **kw)
    rows = B * n
    same("y", y.view(-1, d)[:rows], y64)
    if n_max is None:
        again, _ = vd.vardrop_ffn_fwd(ctx, x, g["W1"], g["W2"], g["b1"], g["b2"], act=vd.ACT_RELU, train=False, ws=ws)
        assert torch.equal(again, y)
    ws.fill_(0xFF)
    grads, more = rooms((d, f), (f, d), (f,), (d,), dtype=gt)
    vd.vardrop_ffn_bwd(ctx, dy, g["W1"], g["W2"], saved, act=vd.ACT_RELU, ws=ws, out=(dx, *grads), **kw)
    for name, got in zip(NAMES, (dx, *grads)):
        same(name, got.view(-1, d)[:rows] if name == "dx" else got, want[name])
    for end in (*ends, *more, y.view(-1)[rows * d:], dx.view(-1)[rows * d:]):
        assert bool((end == 7.0).all())
    assert not kw or int(kw["status"]) == 0


@pytest.mark.parametrize("B,n,d,f", list(u.LARGE))
def test_whole_numbers_in_bf16(vd, ctx, B, n, d, f):
    whole_block(vd, ctx, B, n, d, f, BF16, F32 if d < f else BF16)


@pytest.mark.parametrize("B,n,d,f", list(u.LARGE_FP32))
def test_whole_numbers_in_fp32(vd, ctx, B, n, d, f):
    whole_block(vd, ctx, B, n, d, f, F32, F32)


@pytest.mark.parametrize("dt,B,n,n_max,d,f", [(BF16, 3, 4001, 10003, 448, 1600), (BF16, 1, 6999, 7001, 1984, 2112), (BF16, 1, 65, 16001, 832, 1984),
                                              (F32, 1, 777, 6001, 450, 500)])
def test_whole_numbers_and_a_count_on_the_device(vd, ctx, dt, B, n, n_max, d, f):
    """The tiles of the bound, in the middle of which the tokens end."""
    assert (B, n_max, d, f) in {**u.LARGE, **u.LARGE_FP32}
    whole_block(vd, ctx, B, n, d, f, dt, F32, n_max=n_max)


def rounded(x, ex, dt):
    return ex if dt is F32 else ex + BF * (x.abs() + ex)


def within(name, got, want, bound, norm=2.0 ** -7):
    diff = (got.to(u.F64).reshape(want.shape) - want).abs()
    assert bool((diff <= bound).all()), "%s: %.3g of the bound" % (name, float((diff / bound).max()))
    assert float(diff.norm()) <= norm * float(want.norm()), "%s: off by %.3g of its norm" % (name, float(diff.norm() / want.norm()))


@pytest.mark.parametrize("B,n,d,f", [(1, 16001, 832, 1984), (3, 10003, 448, 1600)])
def test_gelu_in_large_tiles(vd, ctx, B, n, d, f):
    """Bounds as util_ffn.py follows them, y and dh with GELU as it stands in the bf16 kernels."""
    t = {k: None if v is None else v.to(BF16) for k, v in u.dense(B * n, d, f).items()}
    w = u.wide(t)

    def product(A, M, eA=None):
        A, M = A.abs(), M.abs()
        e = A @ M * ((A.shape[-1] + 4) * 2 * U)
        return e if eA is None else e + eA @ M

    def act_error(x, ex, rise):
        tail = u.cdf(-x.abs()) * (2.7e-5 + 200 * U)
        own = (tail + 1.5e-5 + 6e-7 if rise else x.abs() * tail + 1.1e-7) + 8 * U * (1 + x.abs())
        return own + (0.8 if rise else 1.13) * ex

    y, h = u.forward(w, "gelu")
    a = u.act("gelu", h)
    eh = product(w["x"], w["W1"]) + 2 * U * (h.abs() + w["b1"].abs())
    ey = product(a, w["W2"], rounded(a, act_error(h, eh, False), BF16)) + 2 * U * (y.abs() + w["b2"].abs())
    got, saved = vd.vardrop_ffn_fwd(ctx, t["x"].view(B, n, d), t["W1"], t["W2"], t["b1"], t["b2"])
    within("y", got, y, rounded(y, ey, BF16))
    del y, ey, a, got
    first = vd.vardrop_pack8_bytes(B, n, d)
    kx = vd.vardrop_unpack8(ctx, saved[:first], torch.empty(B, n, d, device="cuda")).to(u.F64).view(-1, d)
    kh = vd.vardrop_unpack8(ctx, saved[first:], torch.empty(B, n, f, device="cuda")).to(u.F64).view(-1, f)
    assert torch.equal(kx, u.pack(w["x"])[2])
    most = torch.nn.functional.pad(h.abs() + eh, (0, -f % 32)).view(B * n, -1, 32).amax(-1).repeat_interleave(32, 1)[:, :f]
    assert bool(((kh - h).abs() <= eh + most * 2.0 ** -7 * 1.005).all())
    del h, eh, most
    want = u.backward(w, kx, kh, "gelu")
    da, rise, a = w["dy"] @ w["W2"].t(), u.slope("gelu", kh), u.act("gelu", kh)
    dh = da * rise
    edh = product(w["dy"], w["W2"].t()) * (rise.abs() + U) + da.abs() * act_error(kh, 0.0, True) + 2 * U * dh.abs()
    edh = rounded(dh, edh, BF16)
    ea = rounded(a, act_error(kh, 0.0, False), BF16)
    T = B * n
    e = dict(dx=rounded(want["dx"], product(dh, w["W1"].t(), edh), BF16), dW1=product(kx.t(), dh) + kx.abs().t() @ edh,
             dW2=product(a.t(), w["dy"], ea.t()), db1=edh.sum(0) + 2 * T * U * dh.abs().sum(0), db2=2 * T * U * w["dy"].abs().sum(0))
    out = vd.vardrop_ffn_bwd(ctx, t["dy"].view(B, n, d), t["W1"], t["W2"], saved, bias_grads=True)
    for name, got in zip(NAMES, out):
        within(name, got, want[name], e[name])


# ---- fp32 by parts
def from_checkpoints(vd, ctx, t, T, d, f, kind):
    """The gradients from x and h as 8 bits hold them, and those of the definition."""
    first = vd.vardrop_pack8_bytes(1, T, d)
    saved = torch.zeros(vd.vardrop_ffn_saved_bytes(1, T, d, f), dtype=torch.uint8, device="cuda")
    vd.vardrop_pack8(ctx, t["x"].view(1, T, d), out=saved[:first])
    vd.vardrop_pack8(ctx, t["h"].view(1, T, f), out=saved[first:])
    x, h = u.pack(t["x"])[2], u.pack(t["h"])[2]
    got = vd.vardrop_ffn_bwd(ctx, t["dy"].view(1, T, d), t["W1"], t["W2"], saved, act=vd.ACT_RELU if kind == "relu" else vd.ACT_GELU, bias_grads=True)
    return dict(zip(NAMES, got)), u.backward(u.wide(t), x, h, kind), h


@pytest.mark.parametrize("shift", [0, 1, 77])
@pytest.mark.parametrize("B,T,d,f", list(u.PARTS))
def test_single_products(vd, ctx, B, T, d, f, shift):
    t = u.single_forward(T, d, f, shift)
    want = u.forward(u.wide(t), "relu")[0]
    got = vd.vardrop_ffn_fwd(ctx, t["x"].view(1, T, d), t["W1"], t["W2"], act=vd.ACT_RELU)[0]
    within("y", got, want, 11 * U * want.abs())
    t = u.single_backward(T, d, f, shift)
    got, want, _ = from_checkpoints(vd, ctx, t, T, d, f, "relu")
    within("dx", got["dx"], want["dx"], 11 * U * want["dx"].abs())
    within("dW1", got["dW1"], want["dW1"], 8 * U * want["dW1"].abs())
    t = u.single_dW2(T, d, f, shift)
    got, want, h = from_checkpoints(vd, ctx, t, T, d, f, "gelu")
    within("dW2", got["dW2"], want["dW2"], u.dW2_bound(h, t["dy"].to(u.F64), want["dW2"]))


@pytest.mark.parametrize("B,n,d,f", list(u.LARGE_FP32))
def test_dense_products_by_norm(vd, ctx, B, n, d, f):
    T = B * n
    t = u.dense(T, d, f)
    y = vd.vardrop_ffn_fwd(ctx, t["x"].view(1, T, d), t["W1"], t["W2"], t["b1"], t["b2"])[0]
    assert u.off(y.view(T, d), u.forward(u.wide(t), "gelu")[0]) <= u.norm_bound(d, f)
    got, want, _ = from_checkpoints(vd, ctx, t, T, d, f, "gelu")
    assert u.off(got["dx"].view(T, d), want["dx"]) <= u.norm_bound(d, f)
    if T <= 600:
        assert u.off(got["dW1"], want["dW1"]) <= u.norm_bound(d, T) and u.off(got["dW2"], want["dW2"]) <= u.norm_bound(T)


# ---- 8-bit products
def codes_of(rows):
    """fp32 operations, each rounded once: (codes, scale)."""
    most = rows.float().abs().amax(1)
    up = 127.0 * (1.0 / most)
    return torch.round(rows.float() * up[:, None]).to(torch.int8), most / torch.full_like(most, 127.0)


@pytest.mark.parametrize("kind", ["none", "relu", "gelu"])
@pytest.mark.parametrize("rows,K,N", list(u.LARGE_I8))
def test_8_bit_products(vd, ctx, rows, K, N, kind):
    """The sum is exact; its conversion, two scales and the bias are 6 u of the magnitudes, a result in bf16 is rounded once more."""
    g = u.generator(6, rows, K, N)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    for dt in (BF16, F32):
        x, W, b = (normal(rows, K) * normal(rows, 1).exp()).to(dt), (normal(K, N) * normal(N).exp() * K ** -0.5).to(dt), normal(N).to(dt)
        codes, scale = vd.vardrop_quantize_weight(ctx, W)
        given = vd.vardrop_quantize_rows(ctx, x)
        q, s = codes_of(x)
        w, c = codes_of(W.t().contiguous())
        for have, want in ((given, (q, s)), ((codes, scale), (w, c))):
            assert torch.equal(have[0][:, :K], want[0]) and not bool(have[0][:, K:].any()) and torch.equal(have[1], want[1])
        v = q.to(u.F64) @ w.to(u.F64).t() * (s.to(u.F64)[:, None] * c.to(u.F64))
        e = 6 * U * (v.abs() + b.to(u.F64).abs())
        v = v + b.to(u.F64)
        want = v if kind == "none" else u.act(kind, v)
        if kind == "gelu":
            own = 8 * U * (1 + v.abs()) + (0 if dt is F32 else v.abs() * u.cdf(-v.abs()) * (2.7e-5 + 200 * U) + 1.1e-7)
            e = 1.13 * e + own
        (y,), ends = rooms((rows, N), dtype=dt)
        act = {"none": vd.ACT_NONE, "relu": vd.ACT_RELU, "gelu": vd.ACT_GELU}[kind]
        vd.vardrop_linear_i8(ctx, x, codes, scale, b, act=act, out=y)
        within("y", y, want, rounded(want, e, dt))
        assert bool((ends[0] == 7.0).all())
        assert torch.equal(vd.vardrop_linear_i8(ctx, given, codes, scale, b, act=act), y)


# ---- 8-bit checkpoints past one turn of the grid
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("n,d", [(65536, 768), (65521, 321), (140001, 33)])
def test_checkpoints_of_many_rows(vd, ctx, n, d, dt):
    """More than 33.5 million elements in whole blocks, more than 131 072 blocks of any width: workgroups take several turns."""
    assert n * d > 4096 * 1024 * 8 if d % 32 == 0 else n * -(-d // 32) > 2 * 4096 * 32
    g = u.generator(7, n, d)
    x = (torch.randn(n, d, generator=g, device="cuda") * torch.randn(n, 1, generator=g, device="cuda").exp()).to(dt)
    size = vd.vardrop_pack8_bytes(1, n, d)
    room = torch.full((size + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    saved = vd.vardrop_pack8(ctx, x.view(1, n, d), out=room[:size])
    codes, exps, values = u.pack(x)
    at = -(-n * d // 256) * 256
    assert torch.equal(saved[:n * d].view(torch.int8).view(n, d), codes)
    assert torch.equal(saved[at:at + exps.numel()].view(exps.shape), exps) and bool((room[size:] == 0xAB).all())
    for other in (BF16, F32):
        (back,), ends = rooms((1, n, d), dtype=other)
        vd.vardrop_unpack8(ctx, saved, back)
        assert torch.equal(back.view(n, d).to(u.F64), values) and bool((ends[0] == 7.0).all())


# ---- what is not finite
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("kind", ["relu", "gelu"])
def test_what_is_not_finite_reaches_every_sum_over_its_tokens(vd, ctx, kind, dt):
    """A token with a NaN or an infinity has no h that is a number: its rows of y and dx, and dW1, dW2 and db1, which add its row up, are NaN throughout; the others and db2
    are those of the same call without it."""
    T, d, f = 200, 128, 192
    t = {k: v.to(dt) for k, v in u.dense(T, d, f).items()}
    act = vd.ACT_RELU if kind == "relu" else vd.ACT_GELU

    def both(x):
        y, saved = vd.vardrop_ffn_fwd(ctx, x.view(1, T, d), t["W1"], t["W2"], t["b1"], t["b2"], act=act)
        dx, *rest = vd.vardrop_ffn_bwd(ctx, t["dy"].view(1, T, d), t["W1"], t["W2"], saved, act=act, bias_grads=True)
        return y[0], dx[0], dict(zip(NAMES[1:], rest))

    y, dx, rest = both(t["x"])
    spoilt = t["x"].clone()
    spoilt[7, 3], spoilt[130, 5] = float("nan"), float("inf")
    y2, dx2, rest2 = both(spoilt)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[[7, 130]] = True
    assert not bool(torch.isfinite(y2[bad]).any()) and torch.equal(y2[~bad], y[~bad])
    assert bool(torch.isnan(dx2[bad]).all()) and torch.equal(dx2[~bad], dx[~bad])
    for name in ("dW1", "dW2", "db1"):
        assert bool(torch.isnan(rest2[name]).all()), name
    assert torch.equal(rest2["db2"], rest["db2"]) and bool(torch.isfinite(rest["db2"]).all())


@pytest.mark.parametrize("shape", [(6, 200), (2, 3, 200), (3, 1, 2, 200), (700, 200)])
def test_given_codes_of_any_rank(vd, ctx, shape):
    """Rows of codes viewed as a batch give the rows of the plain call."""
    g = u.generator(8, *shape)
    x, W = torch.randn(shape, generator=g, device="cuda"), torch.randn(shape[-1], 40, generator=g, device="cuda")
    weight = vd.vardrop_quantize_weight(ctx, W)
    q, s = vd.vardrop_quantize_rows(ctx, x)
    want = vd.vardrop_linear_i8(ctx, x, *weight)
    got = vd.vardrop_linear_i8(ctx, (q.view(*shape[:-1], -1), s), *weight, dtype=F32)
    assert got.shape == (s.numel(), 40) and torch.equal(got, want.view(-1, 40))
    with pytest.raises(TypeError):
        vd.vardrop_linear_i8(ctx, (q[:, :100].contiguous(), s), *weight)
    if len(shape) > 2:
        with pytest.raises(TypeError):
            vd.vardrop_linear_i8(ctx, (q.view(*shape[:-1], -1), s[:shape[0]]), *weight)
