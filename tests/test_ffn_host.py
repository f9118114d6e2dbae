"""Host side of the feed-forward block and the 8-bit products: sizes, refusals, and how near the fitted GELU of the bf16 kernels is."""
import os
import re

import numpy as np
import pytest

import paper_2501_14183_amd as vd
from oracle import feedforward as o

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    return vd.load_library()


def fitted(name):
    """Coefficients of a polynomial in pack8.h, highest power first."""
    text = open(os.path.join(ROOT, "paper_2501_14183_amd", "csrc", "pack8.h")).read()
    body = re.search(r"inline float %s\(float u\) \{(.*?)\n\}" % name, text, re.S).group(1)
    return [np.float32(v) for v in re.findall(r"(-?\d+\.\d+(?:e-\d+)?)f", body)]


def horner(coefficients, u):
    """In fp32 with fused products, as the kernels form it."""
    p = np.full_like(u, coefficients[0])
    for c in coefficients[1:]:
        p = (p.astype(np.float64) * u + c).astype(np.float32)
    return p.astype(np.float64)


def test_the_fits_of_gelu():
    u = np.linspace(0.0, 5.5, 20001).astype(np.float32)
    w = u.astype(np.float64)
    tail = o.cdf(-w)
    q = np.exp2(horner(fitted("tail_of"), u))
    assert np.abs(q / tail - 1).max() <= 2.7e-5 + 200 * 2.0 ** -24 and len(fitted("tail_of")) == 7
    assert np.abs(w * (q - tail)).max() <= 3.9e-6
    s = tail - w * np.exp(-0.5 * w * w) / np.sqrt(2 * np.pi)
    assert np.abs(horner(fitted("slope_factor"), u) * q - s).max() <= 1.5e-5 and len(fitted("slope_factor")) == 6
    assert 5.5 * tail[-1] <= 1.1e-7 and abs(s[-1]) <= 6e-7


def test_the_fine_fit_of_gelu():
    """Its error over every argument, with t and the exponential off by one step of fp32 either way: below the 8 2^-24 (1 + |x|) that the tests of the fp32 block count."""
    text = open(os.path.join(ROOT, "paper_2501_14183_amd", "csrc", "pack8.h")).read()
    body = re.search(r"inline float fine_tail\(float u, float& power\) \{(.*?)\n\}", text, re.S).group(1)
    c = [np.float32(v) for v in re.findall(r"(-?\d+\.\d+(?:e-\d+)?)f", body)]
    assert c[0] == 0.25 and abs(c[1] + 0.5 / np.log(2)) < 1e-7 and len(c) == 12
    f, x = np.float32, np.linspace(-20, 20, 400001).astype(np.float32)
    w = x.astype(np.float64)
    u = np.minimum(np.abs(x), f(14))
    phi, cdf = np.exp(-0.5 * w * w) / np.sqrt(2 * np.pi), o.cdf(w)
    for step in (-1, 0, 1):
        t = f(1.0 / f(u.astype(np.float64) * 0.25 + 1.0))
        t = np.nextafter(t, f(9 * step)) if step else t
        power = f(np.exp2((u * u * c[1]).astype(np.float64)))
        power = np.nextafter(power, f(9 * step)) if step else power
        q = f(power * horner(c[2:], t))
        value = f(np.maximum(w, 0.0) - u.astype(np.float64) * q)
        s = f(f(u * f(-0.39894228040143268)).astype(np.float64) * power + q)
        slope = np.where(x > 0, f(1.0 - s.astype(np.float64)), s)
        assert (np.abs(value - w * cdf) / (1 + np.abs(w))).max() <= 2 * 2.0 ** -24
        assert (np.abs(slope - cdf - w * phi) / (1 + np.abs(w))).max() <= 7 * 2.0 ** -24


def test_sizes(lib):
    assert lib.vardrop_pack8_bytes(1, 1, 1) == 512 and lib.vardrop_pack8_bytes(2, 4, 64) == 512 + 256
    assert lib.vardrop_pack8_bytes(3, 5, 33) == 512 + 256 and lib.vardrop_pack8_bytes(0, 4, 64) == 0
    assert lib.vardrop_ffn_saved_bytes(4, 10, 64, 128) == lib.vardrop_pack8_bytes(4, 10, 64) + lib.vardrop_pack8_bytes(4, 10, 128)
    for bad in ((-1, 1, 8), (1, -1, 8), (1, 1, 0), (1 << 16, 1 << 15, 8), (1, 1, (1 << 20) + 1)):
        assert lib.vardrop_pack8_bytes(*bad) == 0
    assert [lib.vardrop_i8_pitch(k) for k in (0, 1, 128, 129, 65536, 65537, -3)] == [0, 128, 128, 256, 65536, 0, 0]
    assert lib.vardrop_linear_i8_workspace_bytes(3, 129, 7) == 768 + 256 and lib.vardrop_linear_i8_workspace_bytes(3, 70000, 7) == 0
    size = lib.vardrop_ffn_workspace_bytes
    assert size(1, 8, 64, 100, vd.BF16) == 0 and size(1, 8, 72, 64, vd.BF16) == 0 and size(1, 8, 72, 100, vd.F32) > 0
    assert size(1, 8, 65536, 64, vd.F32) > 0 and size(1, 8, 65600, 64, vd.F32) == 0 and size(1 << 15, 1 << 10, 1, 1, vd.F32) == 0
    assert size(1, 8, 64, 64, vd.I8) == 0 and size(1 << 15, 1 << 15, 64, 64, vd.BF16) == 0


def test_a_workspace_serves_fewer_tokens(lib):
    for dtype in (vd.F32, vd.BF16):
        for d, f in ((64, 64), (128, 512), (512, 2048)):
            sizes = [lib.vardrop_ffn_workspace_bytes(4, n, d, f, dtype) for n in range(0, 3000, 37)]
            assert sizes == sorted(sizes)


def test_no_context_is_refused(lib):
    n = None
    assert lib.vardrop_pack8(n, n, 1, 1, 8, 0, n, n) == -1 and lib.vardrop_unpack8(n, n, 1, 1, 8, 0, n, n) == -1
    assert lib.vardrop_pack8_dev(n, n, 1, n, 1, n, 8, 0, n, n) == -1 and lib.vardrop_unpack8_dev(n, n, 1, n, 1, n, 8, 0, n, n) == -1
    assert lib.vardrop_ffn_fwd(n, n, 1, 1, 64, 64, 1, 2, n, n, n, n, n, n, n, 0, n) == -1
    assert lib.vardrop_ffn_bwd(n, n, 1, 1, 64, 64, 1, 2, n, n, n, n, n, n, n, n, 0, n, 0, n) == -1
    assert lib.vardrop_ffn_fwd_dev(n, n, 1, n, 1, n, 64, 64, 1, 2, n, n, n, n, n, n, n, 0, n) == -1
    assert lib.vardrop_ffn_bwd_dev(n, n, 1, n, 1, n, 64, 64, 1, 2, n, n, n, n, n, n, n, n, 0, n, 0, n) == -1
    assert lib.vardrop_quantize_rows(n, n, 1, 8, 0, n, n, n) == -1 and lib.vardrop_quantize_weight(n, n, 8, 8, 0, n, n, n) == -1
    assert lib.vardrop_linear_i8(n, n, n, 1, 8, 8, 0, n, n, n, 0, n, 0, n, 0, n) == -1


def test_tensors_that_are_not_on_the_gpu_are_refused(lib):
    import torch

    class Ctx:
        _lib, handle = lib, None

    x, W = torch.zeros(1, 2, 64), torch.zeros(64, 64)
    for call in (lambda: vd.vardrop_pack8(Ctx, x), lambda: vd.vardrop_unpack8(Ctx, torch.zeros(512, dtype=torch.uint8), x),
                 lambda: vd.vardrop_ffn_fwd(Ctx, x, W, W), lambda: vd.vardrop_ffn_bwd(Ctx, x, W, W, torch.zeros(2048, dtype=torch.uint8)),
                 lambda: vd.vardrop_quantize_rows(Ctx, x), lambda: vd.vardrop_quantize_weight(Ctx, W),
                 lambda: vd.vardrop_linear_i8(Ctx, x, torch.zeros(64, 128, dtype=torch.int8), torch.zeros(64))):
        with pytest.raises(TypeError):
            call()


def test_kernel_ids_have_names(lib):
    names = [vd.vardrop_kernel_name(k) for k in range(64)]
    for name in ("pack8", "unpack8", "ffn_up", "ffn_down", "ffn_dh", "ffn_grads", "ffn_split", "quantize", "linear_i8"):
        assert names.count(name) == 1
