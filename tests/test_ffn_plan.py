"""Which tiles the sizes of the feed-forward block's tests select, by the rules of csrc/ffn.h and csrc/tile_gemm.h compiled here for the host, and that
the tests of single and dense fp32 products see every pair of parts: on the CPU, with products that leave one out."""
import os
import subprocess

import pytest
import torch

import util_ffn_tiles as u

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include "%s/paper_2501_14183_amd/csrc/ffn.h"
int main() {
  char kind[8];
  long long T;
  int d, f;
  while (std::scanf("%%7s %%lld %%d %%d", kind, &T, &d, &f) == 4) {
    if (kind[0] == 'i') {
      std::printf("%%d\n", product_shape(kRowShapes, T, f, (d + 127) / 128 * 128 / 2));
    } else if (kind[0] == 'b') {
      const GradPlan p = plan_grads(kShapes, T, d, f);
      std::printf("%%d %%d %%d %%d\n", product_shape(kRowShapes, T, f, d), product_shape(kShapes, T, d, f), p.shape, p.slices);
    } else {
      const int D = (d + 63) / 64 * 64, F = (f + 63) / 64 * 64;
      const GradPlan p = plan_grads(kPartShapes, T, D, F, kLeastSlice / 4, 6, 4.5);
      std::printf("%%d %%d %%d %%d\n", product_shape(kPartShapes, T, F, 6 * D), product_shape(kPartShapes, T, D, 6 * F), p.shape, p.slices);
    }
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    path = tmp_path_factory.mktemp("plan")
    (path / "plan.cpp").write_text(PROGRAM % ROOT)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-Wno-unused-command-line-argument",
                    str(path / "plan.cpp"), "-o", str(path / "plan")], check=True, capture_output=True, text=True)

    def ask(kind, cases):
        lines = "".join("%s %d %d %d\n" % (kind, *c) for c in cases)
        out = subprocess.run([str(path / "plan")], input=lines, check=True, capture_output=True, text=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]

    return ask


def by_tokens(cases):
    return [(B * n, d, f) for B, n, d, f in cases]


def test_tiles_of_the_tested_sizes(plan):
    assert plan("bf16", by_tokens(u.LARGE)) == list(u.LARGE.values())
    for cases in (u.LARGE_FP32, u.PARTS):
        assert plan("fp32", by_tokens(cases)) == list(cases.values())
    assert [v for v, in plan("i8", u.LARGE_I8)] == list(u.LARGE_I8.values())


def test_every_tile_is_among_them():
    large = list(u.LARGE.values())
    for at in range(3):
        assert {c[at] for c in large} == {0, 1, 2}
    assert {c[3] > 1 for c in large if c[2] == 2} == {False, True}
    assert {c[:3] for c in u.PARTS.values()} == {(0, 0, 0), (1, 1, 1)} and set(u.LARGE_I8.values()) == {0, 1, 2}
    # (a small fp32 block is one launch, without parts)
    assert all(d * f > 8192 for _, _, d, f in (*u.PARTS, *u.LARGE_FP32))


# ---- what is seen of the parts
PAIRS = [(0, 0), (0, 1), (1, 0), (0, 2), (1, 1), (2, 0)]


def parts(t):
    """hi, mid and lo in 64 bits; t is their sum exactly."""
    out, left = [], t.to(u.F64)
    for _ in range(3):
        out.append(left.float().to(torch.bfloat16).to(u.F64))
        left = left - out[-1]
    assert not left.any()
    return out


def product(A, B, lost=(), one=False):
    """A @ B by parts (`one`: A has one), rounded once to fp32; without the pairs `lost`."""
    a, b = ([A.to(u.F64)], parts(B)) if one else (parts(A), parts(B))
    pairs = [(0, k) for k in range(3)] if one else PAIRS
    return sum((a[i] @ b[j] for i, j in pairs if (i, j) not in lost), torch.zeros((), dtype=u.F64)).float()


CPU = (70, 66, 72)            # tokens, d, f


# (in dW1 a checkpoint's value has one part)
@pytest.mark.parametrize("which,lost", [(which, pair) for which in ("up", "down", "dh", "dx", "dW1", "dW2") for pair in (None, *PAIRS)
                                        if which != "dW1" or not pair or pair[0] == 0])
def test_single_products_show_every_pair(which, lost):
    T, d, f = CPU
    here = lambda name: (lost,) if which == name else ()
    if which in ("up", "down"):
        t = u.single_forward(T, d, f, 1, device="cpu")
        got = product(product(t["x"], t["W1"], here("up")), t["W2"], here("down"))
        want = u.forward(u.wide(t), "relu")[0]
        bound = 11 * u.U * want.abs()
    elif which == "dW2":
        t = u.single_dW2(T, d, f, 1, device="cpu")
        h = u.pack(t["h"])[2]
        got = product(u.act("gelu", h).float().t(), t["dy"], (lost,))
        want = u.backward(u.wide(t), u.pack(t["x"])[2], h, "gelu")["dW2"]
        bound = u.dW2_bound(h, t["dy"].to(u.F64), want)
    else:
        t = u.single_backward(T, d, f, 1, device="cpu")
        x = u.pack(t["x"])[2]
        dh = product(t["dy"], t["W2"].t(), here("dh"))
        got = product(x.t(), dh, here("dW1"), one=True) if which == "dW1" else product(dh, t["W1"].t(), here("dx"))
        name = "dW1" if which == "dW1" else "dx"
        want = u.backward(u.wide(t), x, u.pack(t["h"])[2], "relu")[name]
        bound = (8 if name == "dW1" else 11) * u.U * want.abs()
    assert (want != 0).float().mean() > 0.9
    over = ((got.to(u.F64) - want).abs() > bound).to(u.F64).mean()
    assert over == 0 if lost is None else over > 0.05, float(over)


@pytest.mark.parametrize("lost", [(), PAIRS[3:], *[(p,) for p in PAIRS[:3]]])
@pytest.mark.parametrize("d,f", [c[2:] for c in u.LARGE_FP32])
def test_dense_products_show_a_lost_part(d, f, lost):
    """The three small pairs together, or one of the large ones."""
    t = u.dense(300, d, f, device="cpu")
    want, h = u.forward(u.wide(t), "gelu")
    grads = u.backward(u.wide(t), t["x"].to(u.F64), t["h"].to(u.F64), "gelu")
    seen = lambda got, want, *K: u.off(got, want) > u.norm_bound(*K)
    for up, down in ((lost, ()), ((), lost)):
        a = u.act("gelu", (product(t["x"], t["W1"], up) + t["b1"]).to(u.F64)).float()
        assert seen(product(a, t["W2"], down) + t["b2"], want, d, f) == bool(lost)
        dh = (product(t["dy"], t["W2"].t(), up).to(u.F64) * u.slope("gelu", t["h"].to(u.F64))).float()
        assert seen(product(dh, t["W1"].t(), down), grads["dx"], d, f) == bool(lost)
