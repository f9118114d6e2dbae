"""Norms before and after a block (vardrop_block_norm_fwd / bwd) against the fp64 oracle.

Bounds.  u = 2^-24 is the error of one fp32 operation.  Every result is bounded by K u times its magnitude: the same formula
with absolute values in the place of differences and sums, which is what the rounding errors of the terms scale with.  A row's
sums are at most 32 terms in a lane and 9 levels across lanes, and a dozen operations follow: K = 64.  A column sum has, beside
its terms' own errors, one addition for each row of a range and one for each range (under 200 in the tests): K = 256.
Results in bf16 are rounded once more, by at most 2^-8 of their value.
"""
import itertools

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import block_norm as o
from util_gpu import to_dev, torch_dtype

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
K_ROW, K_COLUMN = 64, 256


@pytest.fixture(scope="module")
def vd():
    import paper_2501_14183_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(vd):
    return vd.Context(0)


def make(seed, B, n, d, res, dtype, pre, post, gate, bias=True):
    """Inputs already representable in their types, the oracle gets the same values."""
    rng = np.random.default_rng([0xB10C, seed, B, n, d])
    level = rng.standard_normal(d)
    t = dict(x=wl.quantise(rng.standard_normal((B, n, d)) + level, res),
             f=wl.quantise(0.7 * rng.standard_normal((B, n, d)) + 0.3, dtype),
             dr=wl.quantise(rng.standard_normal((B, n, d)), res), dh=wl.quantise(rng.standard_normal((B, n, d)), dtype))
    vec = lambda at, s, *shape: wl.quantise(at + s * rng.standard_normal(shape), dtype)
    t["w"], t["b"] = (vec(1, 0.2, d), vec(0, 0.1, d) if bias else None) if pre != "none" else (None, None)
    t["wp"], t["bp"] = (vec(1, 0.2, d), vec(0, 0.1, d) if bias else None) if post != "none" else (None, None)
    t["gate"] = {"none": None, "shared": vec(0.5, 0.5, d), "window": vec(0.5, 0.5, B, d)}[gate]
    if pre == "none":
        t["dh"] = None
    return t


def absolute(a):
    return 0.0 if a is None else np.abs(np.asarray(a, dtype=np.float64))


def gate_magnitude(t, B, d):
    return np.abs(o.gate_rows(t["gate"], B, d))


def forward_magnitudes(t, pre, post, alpha, beta, stats, r):
    B, n, d = t["x"].shape
    mag_r = np.abs(alpha * t["x"])
    if t["f"] is not None:
        hat = (absolute(t["f"]) + np.abs(stats[..., 0:1])) * stats[..., 1:2]
        hat = hat * (1 + np.sqrt((hat ** 2).mean(-1, keepdims=True))) if post != "none" else hat
        mag_r = mag_r + np.abs(beta) * gate_magnitude(t, B, d) * ((hat if t["wp"] is None else hat * absolute(t["wp"])) + absolute(t["bp"]))
    hat = (mag_r + mag_r.mean(-1, keepdims=True) * (pre == "layer")) * stats[..., 3:4]
    hat = hat * (1 + np.sqrt((hat ** 2).mean(-1, keepdims=True)))     # error of the deviation: that of every element, in the mean
    return mag_r, (hat if t["w"] is None else hat * absolute(t["w"])) + absolute(t["b"])


def backward_magnitudes(t, pre, post, alpha, beta, stats, r):
    like = t["dr"] if t["dr"] is not None else r
    B, n, d = like.shape
    D = absolute(t["dr"]) * np.ones(like.shape)
    out = {}

    def through(kind, v, hat, inv):
        return v if kind == "none" else inv * (v + v.mean(-1, keepdims=True) + hat * (v * hat).mean(-1, keepdims=True))

    if pre != "none":
        hat = (np.abs(r) + np.abs(stats[..., 2:3])) * stats[..., 3:4]
        dh = absolute(t["dh"])
        out["db"], out["dw"] = dh.sum((0, 1)), (dh * hat).sum((0, 1))
        D = D + through(pre, dh if t["w"] is None else dh * absolute(t["w"]), hat, stats[..., 3:4])
    out["dx"] = np.abs(alpha) * D
    du = np.abs(beta) * gate_magnitude(t, B, d) * D
    if t["f"] is None:
        out["df"] = du
        return out
    hat = (absolute(t["f"]) + np.abs(stats[..., 0:1])) * stats[..., 1:2]
    uu = (hat if t["wp"] is None else hat * absolute(t["wp"])) + absolute(t["bp"])
    out["dbp"], out["dwp"] = du.sum((0, 1)), (du * hat).sum((0, 1))
    dg = (np.abs(beta) * D * uu).sum(1)
    out["dgate"] = dg if np.ndim(t["gate"]) == 2 and len(t["gate"]) == B else dg.sum(0)
    out["df"] = through(post, du if t["wp"] is None else du * absolute(t["wp"]), hat, stats[..., 1:2])
    return out


def close(got, want, magnitude, K, what):
    bf16 = got.dtype == torch.bfloat16
    got = got.detach().double().cpu().numpy().reshape(want.shape)
    bound = K * U * magnitude + (2.0 ** -8 * np.abs(want) if bf16 else 0.0) + 1e-37
    worst = float((np.abs(got - want) / bound).max()) if want.size else 0.0
    assert np.isfinite(got).all() and worst <= 1.0, "%s: %.3g of the bound" % (what, worst)


def run_case(vd, ctx, t, res, dtype, pre, post, alpha=0.9, beta=-0.5, eps=1e-5):
    """Forward and backward against the oracle; the backward gets the kernels' own r and statistics."""
    kinds = {"none": vd.NORM_NONE, "layer": vd.NORM_LAYER, "rms": vd.NORM_RMS}
    td, tr = torch_dtype(dtype), torch_dtype(res)
    dev = {k: None if a is None else to_dev(a, tr if k in ("x", "dr") else td) for k, a in t.items()}
    kw = dict(pre=kinds[pre], post=kinds[post], w=dev["w"], wp=dev["wp"], gate=dev["gate"], alpha=alpha, beta=beta)
    r, h, stats = vd.vardrop_block_norm_fwd(ctx, dev["x"], dev["f"], b=dev["b"], bp=dev["bp"], eps=eps, **kw)
    okw = dict(pre=pre, post=post, w=t["w"], wp=t["wp"], bp=t["bp"], gate=t["gate"], alpha=alpha, beta=beta)
    wr, wh, wstats = o.block_norm_forward(t["x"], t["f"], b=t["b"], eps=eps, **okw)
    mag_r, mag_h = forward_magnitudes(t, pre, post, alpha, beta, wstats, wr)
    close(r, wr, mag_r, K_ROW, "r")
    if pre != "none":
        close(h, wh, mag_h, K_ROW, "h")
    rows = wstats.reshape(-1, 4)
    wide = mag_r.reshape(len(rows), -1)
    mean_err = np.stack([absolute(t["f"]).reshape(len(rows), -1).mean(1) if t["f"] is not None else 0 * rows[:, 0], rows[:, 1],
                         wide.mean(1), rows[:, 3] * (1 + rows[:, 3] * np.sqrt((wide ** 2).mean(1)))], 1)
    if t["f"] is not None:
        mean_err[:, 1] *= 1 + rows[:, 1] * np.sqrt((t["f"].reshape(len(rows), -1) ** 2).mean(1))
    close(stats, rows, mean_err, K_ROW, "stats")

    r64, st64 = r.double().cpu().numpy(), stats.double().cpu().numpy().reshape(wstats.shape)
    got = dict(zip(("dx", "df", "dw", "db", "dwp", "dbp", "dgate"),
                   vd.vardrop_block_norm_bwd(ctx, dev["dr"], dev["dh"], r, dev["f"], stats, bias_grads=True, **backward_kw(vd, kw, dev))))
    want = o.block_norm_backward(t["dr"], t["dh"], r64, t["f"], st64, **okw)
    mag = backward_magnitudes(t, pre, post, alpha, beta, st64, r64)
    for key, g in got.items():
        if key in ("dx", "df") or key in want and g is not None:
            if g is None:
                assert t["f"] is None
                continue
            close(g, want[key].reshape(g.shape), np.broadcast_to(mag[key], want[key].shape).reshape(g.shape),
                  K_ROW if key in ("dx", "df") else K_COLUMN, key)
    return dev, r, h, stats, got


def backward_kw(vd, kw, dev):
    """The backward of bp needs the gate's gradient, so it takes bp too."""
    return {**kw, "bp": dev["bp"]}


TYPES = [("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")]


@pytest.mark.parametrize("pre,post,gate", itertools.product(o.KINDS, o.KINDS, ("none", "shared", "window")))
def test_every_combination(vd, ctx, pre, post, gate):
    for i, (res, dtype) in enumerate(TYPES):
        run_case(vd, ctx, make(i, 3, 5, 40, res, dtype, pre, post, gate, bias=i != 1), res, dtype, pre, post)


@pytest.mark.parametrize("res,dtype", TYPES)
@pytest.mark.parametrize("d", [1, 2, 3, 4, 7, 16, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 321, 512, 515, 640, 767, 768, 769,
                               1000, 1024, 1025, 2047, 2048, 2050, 4095, 4097, 8191, 8192])
def test_widths(vd, ctx, d, res, dtype):
    run_case(vd, ctx, make(d, 2, 3, d, res, dtype, "layer", "rms", "window"), res, dtype, "layer", "rms", eps=1e-3)


@pytest.mark.parametrize("B,n,d", [(1, 1, 64), (1, 1, 768), (1, 2, 2048), (32, 1, 512), (1, 700, 48), (5, 333, 96), (2, 2000, 256), (40, 3, 33),
                                   (3, 1000, 513), (300, 1, 20)])
@pytest.mark.parametrize("gate", ["shared", "window"])
def test_token_counts(vd, ctx, B, n, d, gate):
    run_case(vd, ctx, make(n, B, n, d, "bf16", "bf16", "rms", "layer", gate), "bf16", "bf16", "rms", "layer")


@pytest.mark.parametrize("B,n,d,res,dtype", [(5, 14000, 16, "fp32", "bf16"), (3, 6001, 129, "bf16", "bf16"), (2, 2500, 1100, "fp32", "fp32")])
def test_more_rows_than_groups_of_lanes(vd, ctx, B, n, d, res, dtype):
    """Groups of lanes take several rows, of several windows."""
    run_case(vd, ctx, make(n, B, n, d, res, dtype, "layer", "rms", "window"), res, dtype, "layer", "rms")


def test_rows_that_do_not_vary_or_lie_far_from_zero(vd, ctx):
    """Constant rows (variance 0), zero rows, a level of 1000 deviations, and one huge channel."""
    t = make(3, 1, 5, 320, "fp32", "fp32", "layer", "layer", "shared")
    t["f"][0, 0] = 0.0
    t["f"][0, 1] = 2.5
    t["f"][0, 2] += 700.0
    t["f"][0, 3, 17] = 1e6
    t["x"][0, 4] = 0.0
    t["f"][0, 4] = 0.0
    run_case(vd, ctx, t, "fp32", "fp32", "layer", "layer", eps=1e-3)


def test_first_block_has_no_branch_and_first_gradient_may_be_missing(vd, ctx):
    for res, dtype in TYPES:
        t = make(5, 2, 9, 136, res, dtype, "layer", "none", "none")
        t["f"] = None
        run_case(vd, ctx, t, res, dtype, "layer", "none")
        t = make(6, 2, 9, 136, res, dtype, "rms", "rms", "shared")
        t["dr"] = None
        run_case(vd, ctx, t, res, dtype, "rms", "rms")


def test_a_non_finite_token_stays_in_its_row(vd, ctx):
    t = make(8, 2, 6, 72, "fp32", "fp32", "layer", "rms", "shared")
    t["f"][1, 2, 5], t["x"][0, 3, 71] = np.nan, np.inf
    dev = {k: None if a is None else to_dev(a, torch.float32) for k, a in t.items()}
    r, h, stats = vd.vardrop_block_norm_fwd(ctx, dev["x"], dev["f"], pre=vd.NORM_LAYER, post=vd.NORM_RMS, w=dev["w"], wp=dev["wp"], gate=dev["gate"])
    bad = ~torch.isfinite(h).all(-1)
    assert bad.nonzero().tolist() == [[0, 3], [1, 2]]


def test_results_do_not_depend_on_scheduling_and_may_overwrite_inputs(vd, ctx):
    t = make(9, 4, 500, 192, "bf16", "bf16", "layer", "layer", "window")
    dev, r, h, stats, got = run_case(vd, ctx, t, "bf16", "bf16", "layer", "layer")
    kw = dict(pre=vd.NORM_LAYER, post=vd.NORM_LAYER, w=dev["w"], wp=dev["wp"], bp=dev["bp"], gate=dev["gate"], alpha=0.9, beta=-0.5)
    for _ in range(3):
        again = vd.vardrop_block_norm_bwd(ctx, dev["dr"], dev["dh"], r, dev["f"], stats, bias_grads=True, **kw)
        for a, b in zip(again, got.values()):
            assert torch.equal(a, b)
    x, f = dev["x"].clone(), dev["f"].clone()
    vd.vardrop_block_norm_fwd(ctx, x, f, b=dev["b"], out=(x, f, None), **kw)
    assert torch.equal(x, r) and torch.equal(f, h)
    dr, dh = dev["dr"].clone(), dev["dh"].clone()
    ws = torch.empty(vd.vardrop_block_norm_workspace_bytes(4, 500, 192, 4), dtype=torch.uint8, device="cuda")
    vd.vardrop_block_norm_bwd(ctx, dr, dh, r, dev["f"], stats, ws=ws, out=(dr, dh, None, None, None, None, None), **kw)
    assert torch.equal(dr, got["dx"]) and torch.equal(dh, got["df"])


@pytest.mark.parametrize("gate", ["none", "shared", "window"])
@pytest.mark.parametrize("n,n_max", [(0, 7), (1, 7), (7, 7), (40, 300), (301, 700)])
def test_device_side_count(vd, ctx, n, n_max, gate):
    """The rows of [B, N', d] packed in buffers for n_max: bit-identical rows, column sums within the bound of their order."""
    B, d = 3, 80
    t = make(n, B, max(n, 1), d, "bf16", "bf16", "layer", "rms", gate)
    kw = dict(pre=vd.NORM_LAYER, post=vd.NORM_RMS, alpha=0.9, beta=-0.5)
    dev = {k: None if a is None else to_dev(a, torch.bfloat16) for k, a in t.items()}
    par = {k: dev[k] for k in ("w", "wp", "bp", "gate")}

    def packed(a):
        buf = torch.full((B, n_max, d), 7.0, dtype=a.dtype, device="cuda")
        buf.view(-1)[:B * n * d] = a[:, :n].reshape(-1)
        return buf

    n_dev, status = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    r, h, stats = vd.vardrop_block_norm_fwd(ctx, packed(dev["x"]), packed(dev["f"]), b=dev["b"], n_dev=n_dev, status=status, **par, **kw)
    grads = vd.vardrop_block_norm_bwd(ctx, packed(dev["dr"]), packed(dev["dh"]), r, packed(dev["f"]), stats, bias_grads=True, n_dev=n_dev,
                                      status=status, **par, **kw)
    assert int(status) == 0
    if n == 0:
        for g in grads[2:]:
            assert g is None or not g.any()
        return
    r1, h1, stats1 = vd.vardrop_block_norm_fwd(ctx, dev["x"], dev["f"], b=dev["b"], **par, **kw)
    want = vd.vardrop_block_norm_bwd(ctx, dev["dr"], dev["dh"], r1, dev["f"], stats1, bias_grads=True, **par, **kw)
    for a, b in ((r, r1), (h, h1), (stats, stats1), (grads[0], want[0]), (grads[1], want[1])):
        assert torch.equal(a.reshape(-1)[:b.numel()], b.reshape(-1))
    mag = backward_magnitudes(t, "layer", "rms", 0.9, -0.5, stats1.double().cpu().numpy().reshape(B, n, 4), r1.double().cpu().numpy())
    for key, a, b in zip(("dw", "db", "dwp", "dbp", "dgate"), grads[2:], want[2:]):
        if b is not None:
            assert ((a - b).abs().cpu().numpy() <= 2 * K_COLUMN * U * mag[key].reshape(b.shape)).all()


def test_device_side_count_out_of_range_writes_nothing(vd, ctx):
    B, n_max, d = 2, 6, 64
    x = torch.randn(B, n_max, d, device="cuda")
    for bad in (-1, 7):
        n_dev, status = torch.tensor([bad], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        out = (torch.full_like(x, 3.0), torch.full_like(x, 3.0), torch.full((B * n_max, 4), 3.0, device="cuda"))
        vd.vardrop_block_norm_fwd(ctx, x, x, out=out, n_dev=n_dev, status=status)
        assert int(status) == 1 and all(bool((t == 3.0).all()) for t in out)
        status.zero_()
        w = torch.ones(d, device="cuda")
        grads = (torch.full_like(x, 3.0), torch.full_like(x, 3.0), torch.full((d,), 3.0, device="cuda"), None, None, None, None)
        vd.vardrop_block_norm_bwd(ctx, x, x, x, x, torch.ones(B * n_max, 4, device="cuda"), w=w, out=grads, n_dev=n_dev, status=status)
        assert int(status) == 1 and all(bool((t == 3.0).all()) for t in grads[:3])


def test_empty_batches(vd, ctx):
    for B, n in ((0, 5), (4, 0)):
        x = torch.empty(B, n, 64, device="cuda")
        w = torch.ones(64, device="cuda")
        r, h, stats = vd.vardrop_block_norm_fwd(ctx, x, x, w=w, b=w)
        dx, df, dw, db, *_ = vd.vardrop_block_norm_bwd(ctx, x, x, r, x, stats, w=w, bias_grads=True)
        assert not dw.any() and not db.any() and r.shape == x.shape


def test_difference_of_the_kernels_own_forward(vd, ctx):
    """Central difference of the forward along a random direction.  With step 2^-6 of inputs of size 1 the third derivative
    leaves about 2^-12 of the slope, rounding (2^-24 of 3e4 terms in quadrature, over the step) less."""
    t = make(11, 2, 60, 256, "fp32", "fp32", "layer", "layer", "window")
    dev = {k: to_dev(a, torch.float32) for k, a in t.items()}
    names = ("x", "f", "w", "b", "wp", "bp", "gate")
    kw = dict(pre=vd.NORM_LAYER, post=vd.NORM_LAYER, alpha=0.9, beta=0.5)
    g = torch.Generator(device="cuda").manual_seed(3)
    way = {k: torch.randn(dev[k].shape, device="cuda", generator=g) for k in names}

    def loss(step):
        a = {k: dev[k] + step * way[k] for k in names}
        r, h, _ = vd.vardrop_block_norm_fwd(ctx, a.pop("x"), a.pop("f"), **a, **kw)
        return float((r.double() * dev["dr"]).sum() + (h.double() * dev["dh"]).sum())

    r, h, stats = vd.vardrop_block_norm_fwd(ctx, dev["x"], dev["f"], **{k: dev[k] for k in names[2:]}, **kw)
    grads = vd.vardrop_block_norm_bwd(ctx, dev["dr"], dev["dh"], r, dev["f"], stats, w=dev["w"], wp=dev["wp"], bp=dev["bp"],
                                      gate=dev["gate"], bias_grads=True, **kw)
    order = ("x", "f", "w", "b", "wp", "bp", "gate")
    slope = sum(float((gr.double() * way[k]).sum()) for k, gr in zip(order, grads))
    size = sum(float(gr.double().norm() * way[k].double().norm()) / way[k].numel() ** 0.5 for k, gr in zip(order, grads))
    step = 2.0 ** -6
    assert abs((loss(step) - loss(-step)) / (2 * step) - slope) <= 4e-3 * size


@pytest.mark.parametrize("res,dtype", TYPES)
@pytest.mark.parametrize("B,n,d", [(1, 3, 2), (2, 5, 63), (2, 3, 64), (1, 9, 130), (2, 3, 321), (1, 5, 640), (1, 3, 1500), (1, 2, 4100), (1, 1, 8190)])
def test_tensors_at_any_element_and_neighbours_untouched(vd, ctx, B, n, d, res, dtype):
    """Every tensor a slice, at an odd element, of a buffer of sevens that is still there around the results afterwards."""
    t = make(d, B, n, d, res, dtype, "layer", "rms", "window")
    td, tr = torch_dtype(dtype), torch_dtype(res)
    whole = []

    def inside(shape, dt, values=None):
        count = int(np.prod(shape))
        flat = torch.full((count + 40,), 7.0, dtype=dt, device="cuda")
        view = flat[19:19 + count].view(*shape)
        whole.append((flat, count))
        if values is not None:
            view.copy_(to_dev(values, dt))
        return view

    dev = {k: None if a is None else inside(a.shape, tr if k in ("x", "dr") else td, a) for k, a in t.items()}
    plain = {k: None if a is None else to_dev(a, tr if k in ("x", "dr") else td) for k, a in t.items()}
    kw = dict(pre=vd.NORM_LAYER, post=vd.NORM_RMS, alpha=0.9, beta=-0.5)
    stats = torch.empty(B * n, 4, device="cuda")
    out = (inside((B, n, d), tr), inside((B, n, d), td), stats)
    par = lambda v: {k: v[k] for k in ("w", "wp", "bp", "gate")}
    vd.vardrop_block_norm_fwd(ctx, dev["x"], dev["f"], b=dev["b"], out=out, **par(dev), **kw)
    want = vd.vardrop_block_norm_fwd(ctx, plain["x"], plain["f"], b=plain["b"], **par(plain), **kw)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    f32 = torch.float32
    grads = (inside((B, n, d), tr), inside((B, n, d), td)) + tuple(inside((d,), f32) for _ in range(4)) + (inside((B, d), f32),)
    ws = torch.full((vd.vardrop_block_norm_workspace_bytes(B, n, d, B) + 256,), 9, dtype=torch.uint8, device="cuda")
    vd.vardrop_block_norm_bwd(ctx, dev["dr"], dev["dh"], out[0], dev["f"], stats, ws=ws[:-256], out=grads, **par(dev), **kw)
    want = vd.vardrop_block_norm_bwd(ctx, plain["dr"], plain["dh"], want[0], plain["f"], stats, bias_grads=True, **par(plain), **kw)
    assert all(torch.equal(a, b) for a, b in zip(grads, want))
    assert bool((ws[-256:] == 9).all())
    for flat, count in whole:
        assert bool((flat[:19] == 7.0).all()) and bool((flat[19 + count:] == 7.0).all())


def test_recorded_step_follows_the_device_side_count(vd, ctx):
    """Forward and backward in a graph: every replay, with another count and other data, gives what the calls give."""
    B, n_max, d = 4, 50, 192
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(*s, device="cuda", generator=g)
    x, f, dr, dh = (new(B, n_max, d).to(torch.bfloat16) for _ in range(4))
    w, wp, gate = new(d).to(torch.bfloat16), new(d).to(torch.bfloat16), new(B, d).to(torch.bfloat16)
    kw = dict(pre=vd.NORM_LAYER, post=vd.NORM_LAYER, w=w, wp=wp, gate=gate)
    n_dev = torch.tensor([n_max], dtype=torch.int32, device="cuda")
    ws = torch.empty(vd.vardrop_block_norm_workspace_bytes(B, n_max, d, B), dtype=torch.uint8, device="cuda")

    def buffers():
        return ((torch.zeros_like(x), torch.zeros_like(x), torch.zeros(B * n_max, 4, device="cuda")),
                (torch.zeros_like(x), torch.zeros_like(x), torch.zeros(d, device="cuda"), None, torch.zeros(d, device="cuda"), None,
                 torch.zeros(B, d, device="cuda")))

    def step(out, grads):
        vd.vardrop_block_norm_fwd(ctx, x, f, out=out, n_dev=n_dev, **kw)
        vd.vardrop_block_norm_bwd(ctx, dr, dh, out[0], f, out[2], ws=ws, out=grads, n_dev=n_dev, **kw)

    recorded, called = buffers(), buffers()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*recorded)
    for n in (50, 7, 0, 33, 50, 1):
        n_dev.fill_(n)
        for t in (x, f, dr, dh):
            t.copy_(new(B, n_max, d))
        for t in recorded[0] + recorded[1] + called[0] + called[1]:
            if t is not None:
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        step(*called)
        torch.cuda.synchronize()
        for a, b in zip(recorded[0] + recorded[1], called[0] + called[1]):
            assert a is None or torch.equal(a, b), n


def test_rows_beyond_32_bit_offsets(vd, ctx):
    """2^31 + 1024 elements: the last rows are those of a small batch."""
    d = 512
    n = 2 ** 31 // d + 2
    x = torch.zeros(1, n, d, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(1, 300, d, device="cuda").to(torch.bfloat16)
    x[:, n - 300:] = tail
    r, h, stats = vd.vardrop_block_norm_fwd(ctx, x, want_r=False)
    _, want, wstats = vd.vardrop_block_norm_fwd(ctx, tail, want_r=False)
    assert torch.equal(h[:, n - 300:], want) and torch.equal(stats[n - 300:], wstats)
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    dx, _, dw, *_ = vd.vardrop_block_norm_bwd(ctx, None, h, x, None, stats, w=w)
    wdx, _, wdw, *_ = vd.vardrop_block_norm_bwd(ctx, None, want, tail, None, wstats, w=w)
    assert torch.equal(dx[:, n - 300:], wdx)
    assert torch.allclose(dw, wdw, rtol=1e-5, atol=1e-3)


def test_refusals(vd, ctx):
    x = torch.randn(2, 3, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    fwd = lambda *a, **k: vd.vardrop_block_norm_fwd(ctx, *a, **k)
    for bad in (dict(eps=0.0), dict(eps=float("nan")), dict(alpha=float("inf")), dict(beta=float("nan")), dict(pre=5), dict(post=-1),
                dict(pre=vd.NORM_NONE, w=w), dict(post=vd.NORM_NONE, wp=w)):
        with pytest.raises(vd.VarDropError) as e:
            fwd(x, x, **bad)
        assert e.value.code == -1
    with pytest.raises(vd.VarDropError):
        fwd(x, None, post=vd.NORM_RMS)
    with pytest.raises(vd.VarDropError):
        fwd(x, None, gate=w)
    with pytest.raises(vd.VarDropError):
        fwd(x, x, out=(None, None, None))
    with pytest.raises(vd.VarDropError):
        fwd(x, x, pre=vd.NORM_NONE, out=(x.clone(), x.clone(), None))
    with pytest.raises(vd.VarDropError) as e:
        fwd(torch.zeros(1, 1, 8193, device="cuda"))
    assert e.value.code == -4
    with pytest.raises(vd.VarDropError) as e:
        fwd(x.to(torch.bfloat16), x)
    assert e.value.code == -4
    for bad in (dict(w=torch.ones(63, device="cuda")), dict(w=w.half()), dict(gate=torch.ones(3, 64, device="cuda")),
                dict(w=w.to(torch.bfloat16))):
        with pytest.raises(TypeError):
            fwd(x, x, **bad)
    with pytest.raises(TypeError):
        fwd(x.transpose(0, 1), x.transpose(0, 1).contiguous())
    with pytest.raises(TypeError):
        fwd(x, x[:, :2].contiguous())
    with pytest.raises(TypeError):
        fwd(x, x, stream=torch.cuda.current_stream().cuda_stream)
    r, h, stats = fwd(x, x, w=w)
    bwd = lambda *a, **k: vd.vardrop_block_norm_bwd(ctx, *a, **k)
    for a, k in (((None, None, r, x, stats), {}), ((x, None, r, x, stats), {}), ((x, x, None, x, stats), {}), ((x, x, r, x, None), {}),
                 ((x, x, r, None, stats), dict(post=vd.NORM_RMS)), ((x, x, r, None, stats), dict(gate=w))):
        with pytest.raises(vd.VarDropError) as e:
            bwd(*a, **k)
        assert e.value.code == -1
    with pytest.raises(vd.VarDropError) as e:
        bwd(x, x, r, x, stats, w=w, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -2
