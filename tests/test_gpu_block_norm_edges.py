"""Norms around a block where a value, an argument or a buffer is out of the ordinary: non-finite elements, branches that are not
there, results that overwrite inputs.

Bounds, u = 2^-24: with no norm on either side a gradient is three products (beta g, times wp = 1, times D): 4 u of its value,
and 2^-8 more where it is rounded to bf16.
"""
import numpy as np
import pytest
import torch

from oracle import block_norm as o
from test_gpu_block_norm import K_ROW, TYPES, U, backward_magnitudes, close, forward_magnitudes, make
from util_gpu import to_dev, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vd():
    import paper_2501_14183_amd as m
    return m


@pytest.fixture(scope="module")
def ctx(vd):
    return vd.Context(0)


def on_device(t, res, dtype):
    return {k: None if a is None else to_dev(a, torch_dtype(res if k in ("x", "dr") else dtype)) for k, a in t.items()}


def same_but_for_rounding(got, want, what):
    """Equal where the oracle is not finite, within three products' rounding where it is."""
    bf16 = got.dtype == torch.bfloat16
    got = got.double().cpu().numpy().reshape(want.shape)
    sound = np.isfinite(want)
    assert np.isfinite(got[sound]).all(), "%s: %d elements are not finite" % (what, (~np.isfinite(got[sound])).sum())
    assert (np.abs(got[sound] - want[sound]) <= (4 * U + (2.0 ** -8 if bf16 else 0.0)) * np.abs(want[sound]) + 1e-37).all(), what
    assert np.array_equal(got[~sound], want[~sound], equal_nan=True), what


@pytest.mark.parametrize("gate", ["none", "shared", "window"])
@pytest.mark.parametrize("d", [3, 40, 64, 321, 1100])
@pytest.mark.parametrize("res,dtype", TYPES)
def test_a_branch_gradient_does_not_depend_on_the_branch_without_a_post_norm(vd, ctx, res, dtype, d, gate):
    """df = beta g D whatever f is: an infinite or missing value in f stays out of it."""
    t = make(1, 2, 5, d, res, dtype, "none", "none", gate)
    t["f"][0, 1, d // 2], t["f"][1, 2, 0], t["f"][1, 4, d - 1] = np.inf, np.nan, -np.inf
    dev = on_device(t, res, dtype)
    dx, df, *_ = vd.vardrop_block_norm_bwd(ctx, dev["dr"], None, dev["x"], dev["f"], None, pre=vd.NORM_NONE, gate=dev["gate"], alpha=0.75,
                                           beta=-0.5)
    g = o.gate_rows(t["gate"], 2, d)
    same_but_for_rounding(dx, 0.75 * t["dr"], "dx")
    same_but_for_rounding(df, -0.5 * g * t["dr"], "df")


@pytest.mark.parametrize("d", [3, 40, 64, 321, 1100])
def test_an_infinite_gradient_stays_in_its_element_without_norms(vd, ctx, d):
    t = make(2, 2, 5, d, "fp32", "fp32", "none", "none", "none")
    t["dr"][0, 1, d // 2], t["dr"][1, 2, 0] = np.inf, -np.inf
    dev = on_device(t, "fp32", "fp32")
    dx, df, *_ = vd.vardrop_block_norm_bwd(ctx, dev["dr"], None, dev["x"], dev["f"], None, pre=vd.NORM_NONE, alpha=0.75, beta=0.5)
    same_but_for_rounding(dx, 0.75 * t["dr"], "dx")
    same_but_for_rounding(df, 0.5 * t["dr"], "df")


@pytest.mark.parametrize("gate", ["shared", "window"])
@pytest.mark.parametrize("post", ["none", "rms"])
def test_an_infinite_gradient_makes_an_infinite_gate_gradient_without_a_bias(vd, ctx, post, gate):
    """dg = beta sum D wp hat(f): infinite in one channel where hat(f) is not zero.  A bias that was not given adds nothing to it."""
    t = make(3, 2, 5, 72, "fp32", "fp32", "none", post, gate, bias=False)
    t["dr"][1, 2, 7] = np.inf
    dev = on_device(t, "fp32", "fp32")
    kinds = {"none": vd.NORM_NONE, "rms": vd.NORM_RMS}
    _, _, stats = vd.vardrop_block_norm_fwd(ctx, dev["x"], dev["f"], pre=vd.NORM_NONE, post=kinds[post], wp=dev["wp"], gate=dev["gate"])
    *_, dgate = vd.vardrop_block_norm_bwd(ctx, dev["dr"], None, dev["x"], dev["f"], stats, pre=vd.NORM_NONE, post=kinds[post], wp=dev["wp"],
                                          gate=dev["gate"], beta=0.5)
    got = dgate.cpu().numpy().reshape(-1, 72)
    sign = np.sign(t["f"][1, 2, 7] * (1.0 if t["wp"] is None else t["wp"][7]))
    assert got[-1, 7] == sign * np.inf
    got[-1, 7] = 0.0
    assert np.isfinite(got).all()


@pytest.mark.parametrize("pre", ["layer", "rms"])
def test_a_first_block_without_weights_in_another_type_than_the_residual(vd, ctx, pre):
    """Only the results say that the block is bf16 beside a fp32 residual."""
    t = make(4, 2, 9, 136, "fp32", "bf16", pre, "none", "none")
    t = {**t, **dict.fromkeys(("f", "w", "b", "gate"))}
    dev = on_device(t, "fp32", "bf16")
    kind = {"layer": vd.NORM_LAYER, "rms": vd.NORM_RMS}[pre]
    h, stats = torch.empty(2, 9, 136, dtype=torch.bfloat16, device="cuda"), torch.empty(18, 4, device="cuda")
    got = vd.vardrop_block_norm_fwd(ctx, dev["x"], pre=kind, out=(None, h, stats))
    wr, wh, wstats = o.block_norm_forward(t["x"], pre=pre)
    close(got[1], wh, forward_magnitudes(t, pre, "none", 1.0, 1.0, wstats, wr)[1], K_ROW, "h")
    st = stats.double().cpu().numpy().reshape(2, 9, 4)
    dx = torch.empty_like(dev["x"])
    vd.vardrop_block_norm_bwd(ctx, dev["dr"], dev["dh"], dev["x"], None, stats, pre=kind, out=(dx,) + (None,) * 6)
    want = o.block_norm_backward(t["dr"], t["dh"], t["x"], None, st, pre=pre)
    close(dx, want["dx"], backward_magnitudes(t, pre, "none", 1.0, 1.0, st, t["x"])["dx"], K_ROW, "dx")


@pytest.mark.parametrize("res,dtype", TYPES)
@pytest.mark.parametrize("pre", ["none", "layer"])
@pytest.mark.parametrize("d", [3, 40, 321, 1100])
def test_the_branch_gradient_needs_no_branch_without_a_post_norm_and_a_gate(vd, ctx, res, dtype, pre, d):
    """df = beta D with f not given; with no norm at all df alone says what type the block has."""
    t = make(5, 2, 5, d, res, dtype, pre, "none", "none")
    dev = on_device(t, res, dtype)
    kind = {"none": vd.NORM_NONE, "layer": vd.NORM_LAYER}[pre]
    r, _, stats = vd.vardrop_block_norm_fwd(ctx, dev["x"], dev["f"], pre=kind, w=dev["w"], b=dev["b"], beta=0.5)
    dx, df = torch.empty_like(dev["x"]), torch.empty_like(dev["f"])
    vd.vardrop_block_norm_bwd(ctx, dev["dr"], dev["dh"], r if pre == "layer" else None, None, stats, pre=kind, w=dev["w"], beta=0.5,
                              out=(dx, df) + (None,) * 5)
    r64, st64 = r.double().cpu().numpy(), stats.double().cpu().numpy().reshape(2, 5, 4)
    t["f"] = None
    want = o.block_norm_backward(t["dr"], t["dh"], r64, None, st64, pre=pre, w=t["w"], beta=0.5)
    mag = backward_magnitudes(t, pre, "none", 1.0, 0.5, st64, r64)
    close(dx, want["dx"], mag["dx"], K_ROW, "dx")
    close(df, want["df"], mag["df"], K_ROW, "df")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,n,d", [(2, 5, 3), (3, 700, 40), (2, 333, 128), (4, 90, 321), (2, 41, 1100), (1, 9, 8192)])
def test_results_may_overwrite_the_other_input(vd, ctx, B, n, d, dtype):
    """r over f and h over x, dx over dh and df over dr, as in buffers of their own."""
    t = make(6, B, n, d, dtype, dtype, "layer", "rms", "window")
    dev = on_device(t, dtype, dtype)
    kw = dict(pre=vd.NORM_LAYER, post=vd.NORM_RMS, w=dev["w"], wp=dev["wp"], bp=dev["bp"], gate=dev["gate"], alpha=0.9, beta=-0.5)
    r, h, stats = vd.vardrop_block_norm_fwd(ctx, dev["x"], dev["f"], b=dev["b"], **kw)
    grads = vd.vardrop_block_norm_bwd(ctx, dev["dr"], dev["dh"], r, dev["f"], stats, bias_grads=True, **kw)
    x, f, st = dev["x"].clone(), dev["f"].clone(), torch.empty_like(stats)
    vd.vardrop_block_norm_fwd(ctx, x, f, b=dev["b"], out=(f, x, st), **kw)
    assert torch.equal(f, r) and torch.equal(x, h) and torch.equal(st, stats)
    dr, dh = dev["dr"].clone(), dev["dh"].clone()
    vectors = tuple(torch.empty_like(g) for g in grads[2:])
    ws = torch.empty(vd.vardrop_block_norm_workspace_bytes(B, n, d, B), dtype=torch.uint8, device="cuda")
    vd.vardrop_block_norm_bwd(ctx, dr, dh, r, dev["f"], stats, ws=ws, out=(dh, dr) + vectors, **kw)
    for a, b in zip((dh, dr) + vectors, grads):
        assert torch.equal(a, b)
