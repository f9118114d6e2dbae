"""Gradient norm, clipping and AdamW over tensor lists against the fp64 oracle.

Bounds, u = 2^-24: the norm is rounded once from fp64 sums (u; 2 u taken); a clipped gradient has the errors of the norm, the
sum, the quotient and the product (4 u; 8 u taken) and in bf16 one rounding more (2^-8).  m and v are three operations on terms
with those errors (12 u of their terms' magnitudes); the step adds the corrections, a square root, a quotient and a product to them: 32 u of
the step's magnitude, and 4 u of the weight's own.
"""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import optimiser as o
from util_gpu import to_dev

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def vd():
    import paper_2501_14183_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(vd):
    return vd.Context(0)


def grads_of(sizes, seed, dtypes=("fp32",), scale=1.0):
    rng = np.random.default_rng([0x6A4D, seed])
    host = [wl.quantise(scale * 10.0 ** rng.uniform(-3, 0) * rng.standard_normal(n), dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]
    dev = [to_dev(h.astype(np.float32), torch.bfloat16 if dtypes[i % len(dtypes)] == "bf16" else torch.float32) for i, h in enumerate(host)]
    return host, dev


def norm_close(got, want):
    assert abs(float(got) - want) <= 2 * U * want, (float(got), want)


SIZES = [[1], [3, 0, 5], [4096], [4095, 4097], [1, 2, 3, 4, 5, 6, 7, 8], [12288, 1, 8191], [100] * 130, [300001, 17], [64 * 64, 64, 64, 96 * 64]]


@pytest.mark.parametrize("dtypes", [("fp32",), ("bf16",), ("fp32", "bf16", "bf16")])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "-".join(map(str, s[:4])))
def test_norm_and_clipping(vd, ctx, sizes, dtypes):
    host, dev = grads_of(sizes, len(sizes), dtypes)
    want = o.grad_norm(host)
    out = [torch.full((n,), 9.0, dtype=(torch.bfloat16, torch.float32)[i % 2], device="cuda") for i, n in enumerate(sizes)]
    tensors = vd.TensorList(ctx, dev, clipped=out)
    norm = vd.vardrop_grad_norm(ctx, tensors)
    norm_close(norm, want)
    for max_norm in (0.5 * want, 2.0 * want + 1.0):
        vd.vardrop_clip_grads(ctx, tensors, norm, max_norm)
        s = o.clip_factor(want, max_norm)
        for h, d, c in zip(host, dev, out):
            err = np.abs(c.double().cpu().numpy() - s * h)
            assert (err <= (8 * U + (2.0 ** -8 if c.dtype == torch.bfloat16 else 0)) * np.abs(s * h)).all()
            assert np.array_equal(d.double().cpu().numpy(), h)
        if s == 1.0:
            assert all(torch.equal(d.to(c.dtype), c) for d, c in zip(dev, out))


def test_clipping_in_place(vd, ctx):
    host, dev = grads_of([5000, 7, 4096], 1, ("fp32", "bf16"))
    kept = [d.clone() for d in dev]
    tensors = vd.TensorList(ctx, dev)
    norm = vd.vardrop_grad_norm(ctx, tensors)
    vd.vardrop_clip_grads(ctx, tensors, norm, 1e9)
    assert all(torch.equal(a, b) for a, b in zip(dev, kept))
    vd.vardrop_clip_grads(ctx, tensors, norm, 0.25)
    s = o.clip_factor(o.grad_norm(host), 0.25)
    for h, d in zip(host, dev):
        err = np.abs(d.double().cpu().numpy() - s * h)
        assert (err <= (8 * U + (2.0 ** -8 if d.dtype == torch.bfloat16 else 0)) * np.abs(s * h)).all()


@pytest.mark.parametrize("scale", [1e-35, 1e-20, 1e18, 3e36])
def test_squares_beyond_single_precision(vd, ctx, scale):
    host, dev = grads_of([3000, 11], 2, scale=scale)
    norm_close(vd.vardrop_grad_norm(ctx, vd.TensorList(ctx, dev)), o.grad_norm([d.double().cpu().numpy() for d in dev]))


def test_empty_lists(vd, ctx):
    empty = [torch.empty(0, device="cuda")]
    for grads in ([], empty):
        tensors = vd.TensorList(ctx, grads, params=grads, exp_avg=grads, exp_avg_sq=grads)
        norm = vd.vardrop_grad_norm(ctx, tensors, out=torch.full((1,), 5.0, device="cuda"))
        assert float(norm) == 0.0
        vd.vardrop_clip_grads(ctx, tensors, norm, 1.0)
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        vd.vardrop_adamw_dev(ctx, tensors, torch.full((1,), 0.1, device="cuda"), step, norm=norm, max_norm=1.0)
        assert int(step) == 1


def state_of(sizes, seed, mid):
    rng = np.random.default_rng([0xADA3, seed])
    p = [rng.standard_normal(n).astype(np.float32) for n in sizes]
    m = [(0.1 * rng.standard_normal(n) if mid else np.zeros(n)).astype(np.float32) for n in sizes]
    v = [(0.01 * rng.random(n) if mid else np.zeros(n)).astype(np.float32) for n in sizes]
    return p, m, v


def check_step(host, before, dev, lr, step, decay, factor, beta1, beta2, eps, weights):
    for i, (g, p, m, v) in enumerate(zip(host, *before)):
        wp, wm, wv = o.adamw(p, m, v, g, lr, step, beta1, beta2, eps, decay[i], factor)
        gp, gm, gv = (dev[k][i].double().cpu().numpy() for k in range(3))
        x = np.abs(factor * g)
        mag_m = beta1 * np.abs(m) + (1 - beta1) * x
        assert (np.abs(gm - wm) <= 12 * U * mag_m + 1e-45).all()
        assert (np.abs(gv - wv) <= 16 * U * wv + 1e-37).all()
        moved = lr * mag_m / (1 - beta1 ** step) / (np.sqrt(wv / (1 - beta2 ** step)) + eps)
        assert (np.abs(gp - wp) <= 4 * U * np.abs(p) + 32 * U * moved).all()
        if weights[i] is not None:
            assert torch.equal(weights[i], dev[0][i].to(torch.bfloat16))


@pytest.mark.parametrize("mid", [False, True])
@pytest.mark.parametrize("max_norm", [0.0, 0.3, 1e6])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "-".join(map(str, s[:4])))
def test_adamw(vd, ctx, sizes, max_norm, mid):
    host, grads = grads_of(sizes, 3, ("fp32", "bf16"))
    before = state_of(sizes, 4, mid)
    dev = [[to_dev(a) for a in k] for k in before]
    weights = [torch.empty(n, dtype=torch.bfloat16, device="cuda") if i % 3 != 2 else None for i, n in enumerate(sizes)]
    decay = [0.1 * (i % 2) for i in range(len(sizes))]
    tensors = vd.TensorList(ctx, grads, params=dev[0], exp_avg=dev[1], exp_avg_sq=dev[2], weights=weights, decay=decay)
    step = 40 if mid else 1
    norm = vd.vardrop_grad_norm(ctx, tensors) if max_norm else None
    vd.vardrop_adamw(ctx, tensors, 0.01, step, beta1=0.9, beta2=0.99, eps=1e-7, norm=norm, max_norm=max_norm)
    check_step(host, before, dev, 0.01, step, decay, o.clip_factor(o.grad_norm(host), max_norm), 0.9, 0.99, 1e-7, weights)


def test_device_step_counter_and_rate_in_a_graph(vd, ctx):
    """A recorded step makes the next step at every replay: bit for bit the steps called one by one."""
    sizes = [5000, 96, 64 * 64, 3]
    host, grads = grads_of(sizes, 5)
    before = state_of(sizes, 6, False)
    lists, states = [], []
    for _ in range(2):
        dev = [[to_dev(a) for a in k] for k in before]
        states.append(dev)
        lists.append(vd.TensorList(ctx, grads, params=dev[0], exp_avg=dev[1], exp_avg_sq=dev[2], decay=[0.01] * 4))
    step, rate = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 0.02, device="cuda")
    norm = torch.empty(1, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vd.vardrop_grad_norm(ctx, lists[0], out=norm)
        vd.vardrop_adamw_dev(ctx, lists[0], rate, step, norm=norm, max_norm=0.5)
    for k in range(1, 6):
        rate.fill_(0.02 / k)
        for g in grads:
            g.mul_(1.1)
        graph.replay()
        torch.cuda.synchronize()
        n = vd.vardrop_grad_norm(ctx, lists[1])
        vd.vardrop_adamw(ctx, lists[1], float(rate), k, norm=n, max_norm=0.5)
        assert int(step) == k and torch.equal(n, norm)
        for a, b in zip(states[0], states[1]):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_step_with_non_finite_gradients_is_skipped(vd, ctx, value):
    host, grads = grads_of([4097, 30], 7)
    grads[0][4096] = value
    p, m, v = [[torch.randn_like(g).abs() for g in grads] for _ in range(3)]
    kept = [[t.clone() for t in k] for k in (grads, p, m, v)]
    tensors = vd.TensorList(ctx, grads, params=p, exp_avg=m, exp_avg_sq=v)
    norm = vd.vardrop_grad_norm(ctx, tensors)
    assert not np.isfinite(float(norm))
    status, step = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.full((1,), 9, dtype=torch.int64, device="cuda")
    vd.vardrop_clip_grads(ctx, tensors, norm, 1.0, status=status[0:])
    vd.vardrop_adamw(ctx, tensors, 0.1, 3, norm=norm, max_norm=1.0, status=status[1:])
    vd.vardrop_adamw_dev(ctx, tensors, torch.ones(1, device="cuda"), step, norm=norm, max_norm=0.0, status=status[2:])
    assert status.tolist() == [1, 1, 1] and int(step) == 9
    for a, b in zip((grads, p, m, v), kept):
        assert all(torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0)) for x, y in zip(a, b))
    # the list works again with sound gradients
    grads[0][4096] = 1.0
    norm_close(vd.vardrop_grad_norm(ctx, tensors), o.grad_norm([g.double().cpu().numpy() for g in grads]))


def test_tensors_at_any_element_and_neighbours_untouched(vd, ctx):
    flat = {k: torch.randn(20000, device="cuda").abs().to(dt) for k, dt in
            (("g", torch.bfloat16), ("p", torch.float32), ("m", torch.float32), ("v", torch.float32), ("w", torch.bfloat16), ("c", torch.bfloat16))}
    kept = {k: t.clone() for k, t in flat.items()}
    cuts = [(1, 4099), (4101, 4102), (4105, 13000)]
    part = {k: [t[a:b] for a, b in cuts] for k, t in flat.items()}
    tensors = vd.TensorList(ctx, part["g"], clipped=part["c"], params=part["p"], exp_avg=part["m"], exp_avg_sq=part["v"], weights=part["w"])
    norm = vd.vardrop_grad_norm(ctx, tensors)
    vd.vardrop_clip_grads(ctx, tensors, norm, 1.0)
    vd.vardrop_adamw(ctx, tensors, 0.1, 1, norm=norm, max_norm=1.0)
    inside = torch.zeros(20000, dtype=torch.bool, device="cuda")
    for a, b in cuts:
        inside[a:b] = True
    for k in flat:
        assert torch.equal(flat[k][~inside], kept[k][~inside])
    host = [t.double().cpu().numpy() for t in part["g"]]
    s = o.clip_factor(o.grad_norm(host), 1.0)
    before = [[kept[k][a:b].cpu().numpy() for a, b in cuts] for k in "pmv"]
    check_step(host, before, [part[k] for k in "pmv"], 0.1, 1, [0.0] * 3, s, 0.9, 0.999, 1e-8, part["w"])


def test_the_same_bits_every_time(vd, ctx):
    host, grads = grads_of([3000001, 17, 4096] + [333] * 100, 8)
    tensors = vd.TensorList(ctx, grads)
    first = vd.vardrop_grad_norm(ctx, tensors)
    assert all(torch.equal(vd.vardrop_grad_norm(ctx, tensors), first) for _ in range(20))


def test_a_tensor_beyond_32_bit_offsets(vd, ctx):
    n = 2 ** 31 + 4099
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[-1], g[2 ** 31] = 2.0, 3.0, 6.0
    out = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    tensors = vd.TensorList(ctx, [g], clipped=[out])
    norm = vd.vardrop_grad_norm(ctx, tensors)
    assert float(norm) == 7.0
    vd.vardrop_clip_grads(ctx, tensors, norm, 3.5)
    assert (float(out[0]), float(out[-1]), float(out[2 ** 31])) == (1.0, 1.5, 3.0)


def test_another_stream(vd, ctx):
    host, grads = grads_of([70000, 5], 9)
    tensors = vd.TensorList(ctx, grads)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        vd.vardrop_grad_norm(ctx, tensors, out=out)
    side.synchronize()
    norm_close(out, o.grad_norm(host))
    out.zero_()
    torch.cuda.synchronize()
    vd.vardrop_grad_norm(ctx, tensors, out=out, stream=side.cuda_stream)
    side.synchronize()
    norm_close(out, o.grad_norm(host))


def test_refusals(vd, ctx):
    g = [torch.ones(8, device="cuda")]
    plain = vd.TensorList(ctx, g)
    whole = vd.TensorList(ctx, g, params=[g[0].clone()], exp_avg=[g[0].clone()], exp_avg_sq=[g[0].clone()])
    norm = vd.vardrop_grad_norm(ctx, plain)
    for call in (lambda: vd.vardrop_clip_grads(ctx, plain, norm, 0.0), lambda: vd.vardrop_clip_grads(ctx, plain, None, 1.0),
                 lambda: vd.vardrop_clip_grads(ctx, plain, norm, float("nan")),
                 lambda: vd.vardrop_adamw(ctx, plain, 0.1, 1), lambda: vd.vardrop_adamw(ctx, whole, 0.1, 0),
                 lambda: vd.vardrop_adamw(ctx, whole, -0.1, 1), lambda: vd.vardrop_adamw(ctx, whole, float("nan"), 1),
                 lambda: vd.vardrop_adamw(ctx, whole, 0.1, 1, beta1=1.0), lambda: vd.vardrop_adamw(ctx, whole, 0.1, 1, beta2=-0.1),
                 lambda: vd.vardrop_adamw(ctx, whole, 0.1, 1, eps=0.0), lambda: vd.vardrop_adamw(ctx, whole, 0.1, 1, max_norm=1.0),
                 lambda: vd.vardrop_adamw(ctx, whole, 0.1, 1, norm=norm, max_norm=-1.0),
                 lambda: vd.vardrop_adamw_dev(ctx, whole, None, torch.zeros(1, dtype=torch.int64, device="cuda")),
                 lambda: vd.vardrop_adamw_dev(ctx, whole, norm, None)):
        with pytest.raises(vd.VarDropError) as e:
            call()
        assert e.value.code == -1
    for args in (dict(clipped=[]), dict(clipped=[torch.ones(7, device="cuda")]), dict(params=g, exp_avg=g, exp_avg_sq=[g[0].half()]),
                 dict(clipped=[torch.ones(8, device="cuda", dtype=torch.float64)]), dict(clipped=[torch.ones(8)]),
                 dict(clipped=[torch.ones(16, device="cuda")[::2]]), dict(params=g, exp_avg=g, exp_avg_sq=g, decay=[0.1, 0.2])):
        with pytest.raises(TypeError):
            vd.TensorList(ctx, g, **args)
    for args in (dict(params=g), dict(weights=[None]), dict(decay=[0.1]), dict(params=g, exp_avg=g, exp_avg_sq=g, decay=[float("nan")])):
        with pytest.raises(vd.VarDropError):
            vd.TensorList(ctx, g, **args)


def test_weight_decay_below_the_last_digit_of_one(vd, ctx):
    """A thousand steps without gradients: weights shrink by (1 - lr decay)^1000 with lr decay = 1e-6, whose rounding beside 1 would
    be off by up to 3 %.  Every step rounds a weight once (2^-24, in either direction): 1000 of them stay below 1000 * 2^-24 = 6e-5 in
    all and 2e-6 in the mean of 4096 weights with their roundings in quadrature; 1 % of the decay is 1e-5."""
    p = torch.rand(4096, device="cuda") + 0.5
    before = p.double()
    g, m, v = (torch.zeros_like(p) for _ in range(3))
    tensors = vd.TensorList(ctx, [g], params=[p], exp_avg=[m], exp_avg_sq=[v], decay=[0.01])
    for step in range(1, 1001):
        vd.vardrop_adamw(ctx, tensors, 1e-4, step)
    shrunk = (p.double() / before).mean()
    assert abs(float(shrunk) - (1 - 1e-6) ** 1000) <= 1e-5
