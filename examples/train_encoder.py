"""Trains a small encoder over the kept variate tokens with nothing but this library's calls around one elementwise loss.

Per step, all on one stream and without a host synchronisation (the number of kept tokens stays on the device):

    hash -> sample -> embed the kept windows -> norm
    -> layers x (attention -> post norm, gate, residual and the next norm in one call; with --ffn the same around a feed-forward block,
       whose activations wait for the backward pass in 8 bits) -> loss
    -> the same backwards -> global gradient norm -> AdamW with clipping

The target is what a second encoder with other weights makes of the same windows, so the loss has a zero to go to.

    python examples/train_encoder.py [--steps 200] [--ffn 256]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2501_14183_amd as vd  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
RES_SCALE, BRANCH_SCALE = 1.0, 0.5


def name(stem, k):
    """Name of a weight of block (or norm) k.  Numbers from ten on stand behind an underscore: b1 of block 1 and b of norm 11 would be one name."""
    return "%s%s%d" % (stem, "_" if k > 9 else "", k)


class Encoder:
    """Weights in fp32 with the bf16 copies that the kernels read, and one step's buffers for up to n_max tokens a window.

    The residual stream is fp32, the blocks are bf16: pre norms LayerNorm, post norms RMSNorm with a learned gate."""

    def __init__(self, ctx, B, L, n_max, d, H, layers, seed, train=True, ffn=0):
        self.ctx, self.B, self.L, self.n_max, self.d, self.H, self.layers, self.ffn = ctx, B, L, n_max, d, H, layers, ffn
        # what stands between two norms: a layer's attention, and with `ffn` channels inside its feed-forward block
        self.blocks = [kind for _ in range(layers) for kind in (("attention", "ffn") if ffn else ("attention",))]
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale, at=0.0):
            return torch.randn(*shape, generator=g, device="cuda") * scale + at

        p = {"We": normal(L, d, scale=L ** -0.5), "be": normal(d, scale=0.1), "w0": normal(d, scale=0.1, at=1.0), "b0": normal(d, scale=0.1)}

        def weight(stem, k, t):
            assert name(stem, k) not in p, name(stem, k)
            p[name(stem, k)] = t

        for k, kind in enumerate(self.blocks):
            if kind == "attention":
                for stem in ("Wq", "Wk", "Wv", "Wo"):
                    weight(stem, k, normal(d, d, scale=d ** -0.5))
            else:
                weight("W1", k, normal(d, ffn, scale=d ** -0.5))
                weight("b1", k, normal(ffn, scale=0.1))
                weight("W2", k, normal(ffn, d, scale=ffn ** -0.5))
                weight("b2", k, normal(d, scale=0.1))
            weight("wp", k, normal(d, scale=0.1, at=1.0))
            weight("gate", k, normal(d, scale=0.1, at=0.5))
            weight("w", k + 1, normal(d, scale=0.1, at=1.0))
            weight("b", k + 1, normal(d, scale=0.1))
        self.low = {k: t.to(BF16) for k, t in p.items()}
        self.params = {k: t.float() for k, t in self.low.items()}

        def tokens(dtype):
            return torch.zeros(B, n_max, d, dtype=dtype, device="cuda")

        lib = ctx._lib
        self.xs, self.x0 = tokens(BF16), tokens(F32)
        self.saved_embed = torch.empty(lib.vardrop_embed_saved_bytes(B, n_max, L, vd.BF16), dtype=torch.uint8, device="cuda")
        sizes = {"attention": lib.vardrop_attn_saved_bytes(B, n_max, d, H, vd.BF16),
                 "ffn": vd.vardrop_ffn_saved_bytes(B, n_max, d, ffn) if ffn else 0}
        self.saved = [torch.empty(sizes[kind], dtype=torch.uint8, device="cuda") for kind in self.blocks]
        self.f = [tokens(BF16) for _ in self.blocks]
        # (r, h, statistics) of every norm; the first has no branch and r = x0
        self.norms = [(None if k == 0 else tokens(F32), tokens(BF16), torch.empty(B * n_max, 4, device="cuda")) for k in range(len(self.blocks) + 1)]
        self.ffn_ws = torch.empty(vd.vardrop_ffn_workspace_bytes(B, n_max, d, ffn, BF16), dtype=torch.uint8, device="cuda") if ffn else None
        if not train:
            return
        self.grads = {k: torch.zeros_like(t) for k, t in self.params.items()}
        self.dr, self.df, self.dh = tokens(F32), tokens(BF16), tokens(BF16)
        size = max(lib.vardrop_attn_workspace_bytes(B, n_max, d, H, vd.BF16), lib.vardrop_embed_workspace_bytes(B, n_max, L, d, vd.BF16),
                   vd.vardrop_block_norm_workspace_bytes(B, n_max, d, 1))
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        names = list(self.params)
        moments = [{k: torch.zeros_like(t) for k, t in self.params.items()} for _ in range(2)]
        self.list = vd.TensorList(ctx, [self.grads[k] for k in names], params=[self.params[k] for k in names],
                                  exp_avg=[moments[0][k] for k in names], exp_avg_sq=[moments[1][k] for k in names],
                                  weights=[self.low[k] for k in names],
                                  decay=[0.01 if self.params[k].dim() == 2 else 0.0 for k in names])
        self.norm = torch.zeros(1, device="cuda")
        self.step_dev = torch.zeros(1, dtype=torch.int64, device="cuda")

    def attention(self, k, of=None):
        """Wq, Wk, Wv, Wo of block k, or what `of` has for them."""
        return [(of or self.low)[name(stem, k)] for stem in ("Wq", "Wk", "Wv", "Wo")]

    def feed_forward(self, k, of=None):
        """W1, W2, b1, b2 of block k, or what `of` has for them."""
        return [(of or self.low)[name(stem, k)] for stem in ("W1", "W2", "b1", "b2")]

    def norm_bias(self, k):
        return self.low[name("b", k)]

    def block(self, k, n_dev):
        """self.f[k] from the norm before it."""
        h = self.norms[k][1]
        if self.blocks[k] == "attention":
            vd.vardrop_attn_fwd_dev(self.ctx, h, n_dev, self.n_max, *self.attention(k), self.H, self.f[k], self.saved[k])
        else:
            vd.vardrop_ffn_fwd(self.ctx, h, *self.feed_forward(k), act=vd.ACT_GELU, saved=self.saved[k], ws=self.ffn_ws, out=self.f[k], n_dev=n_dev)

    def block_backward(self, k, n_dev):
        """self.dh and the gradients of block k's weights from self.df."""
        g = self.grads
        if self.blocks[k] == "attention":
            vd.vardrop_attn_bwd_dev(self.ctx, self.df, self.norms[k][1], n_dev, self.n_max, *self.attention(k), self.H, self.saved[k],
                                    self.ws, (self.dh, *self.attention(k, g)))
        else:
            vd.vardrop_ffn_bwd(self.ctx, self.df, *self.feed_forward(k)[:2], self.saved[k], act=vd.ACT_GELU, ws=self.ffn_ws,
                               out=(self.dh, *self.feed_forward(k, g)), n_dev=n_dev)

    def around(self, k):
        """What the norm behind block k - 1 takes: its own weight, and the post norm and gate of that block."""
        kw = dict(pre=vd.NORM_LAYER, w=self.low[name("w", k)])
        if k > 0:
            kw |= dict(post=vd.NORM_RMS, wp=self.low[name("wp", k - 1)], gate=self.low[name("gate", k - 1)], alpha=RES_SCALE,
                       beta=BRANCH_SCALE)
        return kw

    def forward(self, x, sel, n_dev):
        """-> the last norm's output, [B, N', d] packed in a buffer for n_max."""
        ctx, n_max = self.ctx, self.n_max
        vd.vardrop_embed_fwd_dev(ctx, x, sel, n_dev, n_max, self.low["We"], self.low["be"], self.xs, self.saved_embed)
        self.x0.copy_(self.xs)
        vd.vardrop_block_norm_fwd(ctx, self.x0, b=self.norm_bias(0), out=self.norms[0], n_dev=n_dev, **self.around(0))
        res = self.x0
        for k in range(len(self.blocks)):
            self.block(k, n_dev)
            vd.vardrop_block_norm_fwd(ctx, res, self.f[k], b=self.norm_bias(k + 1), out=self.norms[k + 1], n_dev=n_dev,
                                      **self.around(k + 1))
            res = self.norms[k + 1][0]
        return self.norms[-1][1]

    def backward(self, dh, n_dev):
        """All gradients into self.grads, from that of the last norm's output."""
        ctx, n_max, g, dr = self.ctx, self.n_max, self.grads, None
        for k in range(len(self.blocks), 0, -1):
            r, _, stats = self.norms[k]
            out = (self.dr, self.df, g[name("w", k)], g[name("b", k)], g[name("wp", k - 1)], None, g[name("gate", k - 1)])
            vd.vardrop_block_norm_bwd(ctx, dr, dh, r, self.f[k - 1], stats, ws=self.ws, out=out, n_dev=n_dev, **self.around(k))
            dr, dh = self.dr, self.dh
            self.block_backward(k - 1, n_dev)
        vd.vardrop_block_norm_bwd(ctx, dr, dh, self.x0, None, self.norms[0][2], ws=self.ws,
                                  out=(self.dr, None, g["w0"], g["b0"], None, None, None), n_dev=n_dev, **self.around(0))
        self.df.copy_(self.dr)
        vd.vardrop_embed_bwd_dev(ctx, self.df, n_dev, n_max, self.L, self.saved_embed, self.ws, (g["We"], g["be"]))

    def update(self, rate, max_norm, status=None):
        vd.vardrop_grad_norm(self.ctx, self.list, out=self.norm)
        vd.vardrop_adamw_dev(self.ctx, self.list, rate, self.step_dev, norm=self.norm, max_norm=max_norm, status=status)


def loss_and_gradient(h, target, n_dev, B):
    """Mean squared error over the N' tokens of every window, and its gradient; rows behind them are not looked at."""
    d = h.shape[-1]
    count = (n_dev.float() * B * d).clamp(min=1.0)
    inside = (torch.arange(h.numel() // d, device=h.device) < n_dev * B).unsqueeze(1)
    diff = torch.where(inside, h.reshape(-1, d).float() - target.reshape(-1, d).float(), torch.zeros((), device=h.device))
    return diff.square().sum() / count, (2.0 * diff / count).to(h.dtype).reshape(h.shape)


def periods():
    """The profiles' periods, on the device once: a table made there in every step would be a copy that the host waits for."""
    return torch.tensor([24.0, 12.0, 8.0, 48.0], device="cuda")


def windows(B, N, L, seed, table=None):
    """Noisy daily and weekly profiles, [B, N, L]; table: periods(), made here when it is not given."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.arange(L, device="cuda").float() + 24.0 * torch.rand(B, N, 1, generator=g, device="cuda")
    period = (periods() if table is None else table)[torch.randint(4, (1, N, 1), generator=g, device="cuda")]
    return torch.sin(6.2831853 * t / period) + 0.5 * torch.sin(6.2831853 * t / 24.0) + 0.2 * torch.randn(B, N, L, generator=g, device="cuda")


def train(steps=200, B=8, N=96, L=96, d=128, H=2, layers=2, gs=4, rate=2e-3, max_norm=1.0, say=None, ffn=0):
    """-> losses of all steps (one host read, at the end)."""
    ctx = vd.Context(0)
    student = Encoder(ctx, B, L, N, d, H, layers, seed=1, ffn=ffn)
    teacher = Encoder(ctx, B, L, N, d, H, layers, seed=2, train=False, ffn=ffn)
    draw = torch.zeros(1, dtype=torch.int64, device="cuda")
    selection = tuple(torch.zeros(k, dtype=torch.int32, device="cuda") for k in (N, N, 2))
    rate_dev, status = torch.full((1,), rate, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    table, losses = periods(), []
    for step in range(steps):
        x = windows(B, N, L, seed=step, table=table)
        _, hashes, _ = vd.vardrop_hash(ctx, x, 2)
        _, sel, counts = vd.vardrop_sample_dev(ctx, hashes, gs, 1, 1, 42, draw, True, selection)
        n_dev = counts[:1]
        loss, dh = loss_and_gradient(student.forward(x, sel, n_dev), teacher.forward(x, sel, n_dev), n_dev, B)
        student.backward(dh, n_dev)
        student.update(rate_dev, max_norm, status)
        losses.append(loss)
    losses = torch.cat(losses).tolist()
    assert int(status) == 0 and int(student.step_dev) == steps
    if say:
        for step in range(0, steps, max(1, steps // 10)):
            say("step %4d  loss %.5f" % (step, losses[step]))
        say("step %4d  loss %.5f, gradient norm %.4f, %d of %d variates kept" % (steps - 1, losses[-1], float(student.norm), int(n_dev), N))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--ffn", type=int, default=0, help="channels inside the feed-forward blocks (a multiple of 64); 0: attention alone")
    args = ap.parse_args()
    train(args.steps, say=print, ffn=args.ffn)
