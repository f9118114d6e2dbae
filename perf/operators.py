"""Performance cases of what stands around the attention of a training step: the norms before and after a block with its
gate and residual scale, the global norm and clipping of the gradients, and the AdamW update of the weights.

A case is one of four calls ("path"):

  norm_fwd   r = alpha x + beta gate * post(f) and h = pre(r): a block's output f joins the residual stream x, and the next
             block's input h is formed on the way; post and pre are LayerNorm, RMSNorm or nothing; one gate row for all
             tokens or one for each window of the batch
  norm_bwd   its gradients: dx, df, the norms' weights and biases, the gate
  clip       global norm over a model's gradients, and the gradients scaled to it in the type that the optimiser takes
  adamw      global norm, then one AdamW step of all tensors with the clipping inside: moments and weights in fp32, a bf16
             copy of the weights for the matrix cores; with "dev" the step counter and the rate are in device memory

The tensors of a clip or adamw case lie one after the other in flat buffers, as gradient buckets do: an embedding of
windows of L samples, `layers` encoder layers of width d, and `ragged` tensors of odd sizes.
"""
import torch

own = False
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS_NORM, EPS_CLIP = 1e-5, 1e-6
BETA1, BETA2, EPS_ADAM, RATE, DECAY = 0.9, 0.999, 1e-8, 1e-4, 0.01
MOST_TOKENS, MOST_WEIGHTS = 8 * 8192 * 768, 57_000_000


def listed():
    return [
        # The smallest workload of the repository, 10 of 32 variates kept: add and norm in fp32. Launches count.
        norm("norm_fwd_tiny_fp32", "norm_fwd", 4, 10, 64, "fp32", "fp32", "layer", "none"),
        # Kept tokens of Electricity: add and norm as in the paper's backbone, with biases.
        norm("norm_fwd_electricity", "norm_fwd", 32, 65, 512, "bf16", "bf16", "layer", "none"),
        # All 862 variates of Traffic, norms on both sides of the block, residual stream in fp32, a gate for each window.
        norm("norm_fwd_traffic_dense", "norm_fwd", 32, 862, 512, "fp32", "bf16", "rms", "rms", gate="window", alpha=0.9),
        # A width that no vector load divides: 321 tokens of 321 channels.
        norm("norm_fwd_odd", "norm_fwd", 7, 321, 321, "bf16", "bf16", "layer", "layer", gate="shared"),
        # The everyday training shape: kept tokens of Traffic.
        norm("norm_bwd_traffic", "norm_bwd", 32, 87, 512, "bf16", "bf16", "layer", "rms", gate="shared", beta=0.5),
        # A wide model in fp32 whose rows need several wavefronts.
        norm("norm_bwd_wide_fp32", "norm_bwd", 2, 1001, 2048, "fp32", "fp32", "rms", "none", gate="window"),
        # The largest: all 8192 variates of 8 windows at width 768, everything on.
        norm("norm_bwd_stress_dense", "norm_bwd", 8, 8192, 768, "bf16", "bf16", "layer", "layer", gate="window", alpha=0.9, beta=0.5),
        # One layer and the embedding at the Traffic shape: fp32 gradients clipped into the type of the bf16 weights.
        tensors("clip_layer", "clip", 1, 512, 96, 0, "fp32", "bf16", max_norm=0.5),
        # Hundreds of tensors of an odd width and of odd sizes.
        tensors("clip_ragged", "clip", 24, 321, 97, 300, "fp32", "fp32", max_norm=1.0),
        # The update of that one layer, step counter and rate on the device (a recorded training step).
        tensors("adamw_layer", "adamw", 1, 512, 96, 0, "fp32", "bf16", max_norm=0.5, dev=True),
        # bf16 gradients of an odd width, weights kept in fp32 alone, no clipping.
        tensors("adamw_ragged", "adamw", 12, 321, 336, 100, "bf16", "fp32", max_norm=0.0),
        # 24 layers of the largest width.
        tensors("adamw_stack", "adamw", 24, 768, 512, 0, "fp32", "bf16", max_norm=1.0),
    ]


def norm(name, path, B, n, d, res, dtype, pre, post, gate="none", alpha=1.0, beta=1.0, bias=True):
    return dict(name=name, path=path, B=B, n=n, d=d, res=res, dtype=dtype, pre=pre, post=post, gate=gate, alpha=alpha,
                beta=beta, bias=bias)


def tensors(name, path, layers, d, L, ragged, grad, to, max_norm, dev=False):
    return dict(name=name, path=path, layers=layers, d=d, L=L, ragged=ragged, grad=grad, to=to, max_norm=max_norm, dev=dev)


def spread(rng, lo, hi):
    """A whole number of lo..hi, evenly over its logarithm."""
    return min(hi, int(lo * (hi / lo) ** rng.random() + rng.random()))


def draw(rng):
    path = rng.choice(("norm_fwd", "norm_bwd", "clip", "adamw"))
    if path.startswith("norm"):
        d = rng.choice((64, 128, 192, 256, 320, 384, 512, 640, 768, 1024)) if rng.random() < 0.6 else spread(rng, 16, 2048)
        B = spread(rng, 1, 32)
        n = spread(rng, 1, min(8192, MOST_TOKENS // (B * d)))
        res, dtype = rng.choice((("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")))
        c = norm("", path, B, n, d, res, dtype, rng.choice(("layer", "rms")), rng.choice(("none", "layer", "rms")),
                 rng.choice(("none", "shared", "window")), rng.choice((1.0, 0.9)), rng.choice((1.0, 0.5)), rng.random() < 0.5)
    else:
        d = rng.choice((64, 128, 256, 512, 768)) if rng.random() < 0.5 else spread(rng, 33, 768)
        L = rng.choice((96, 97, 336, 512))
        layers = spread(rng, 1, max(1, min(24, MOST_WEIGHTS // (4 * d * d + 9 * d) - 2)))
        c = tensors("", path, layers, d, L, rng.choice((0, 0, spread(rng, 1, 400))), rng.choice(("fp32", "bf16")),
                    rng.choice(("fp32", "bf16")), rng.choice((1.0, 0.05)) if path == "clip" else rng.choice((0.0, 1.0, 0.05)),
                    path == "adamw" and rng.random() < 0.5)
    del c["name"]
    return c


def sizes(case):
    """Element counts of the tensors of a clip or adamw case: the matrices, which the weight decay shrinks, then the rest."""
    d = case["d"]
    odd = [1 + (7919 * (i + 1)) % 2999 for i in range(case["ragged"])]
    return [case["L"] * d] + [d * d] * (4 * case["layers"]), [d] * (1 + 9 * case["layers"]) + odd


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return prepare_norm(case, g) if case["path"].startswith("norm") else prepare_tensors(case, g)


def prepare_norm(c, g):
    B, n, d, dt, res = c["B"], c["n"], c["d"], TYPES[c["dtype"]], TYPES[c["res"]]

    def normal(*shape, scale=1.0, at=0.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(scale).add_(at)

    # Channels of a residual stream differ in level and scale, a few by far.
    level, loud = normal(d, scale=0.5), 1.0 + normal(d).square_()
    s = dict(c, x=(normal(B, n, d) * loud + level).to(res), f=normal(B, n, d, scale=0.7, at=0.1).to(dt),
             w=normal(d, scale=0.2, at=1.0).to(dt), b=normal(d, scale=0.1).to(dt) if c["bias"] else None,
             wp=normal(d, scale=0.2, at=1.0).to(dt) if c["post"] != "none" else None,
             bp=normal(d, scale=0.1).to(dt) if c["bias"] and c["post"] != "none" else None,
             gate={"none": None, "shared": normal(1, d, scale=0.3, at=0.8).to(dt),
                   "window": normal(B, d, scale=0.3, at=0.8).to(dt)}[c["gate"]])

    def empty(like, *shape):
        return None if like is None else torch.empty(*shape, dtype=torch.float32, device="cuda")

    if c["path"] == "norm_fwd":
        s["out"] = (torch.empty_like(s["x"]), torch.empty_like(s["f"]), empty(level, B * n, 4))
    else:
        s["r"], _, s["stats"] = norm_forward(s)
        s["dr"], s["dh"] = normal(B, n, d, scale=0.01).to(res), normal(B, n, d, scale=0.01).to(dt)
        s["out"] = (torch.empty_like(s["x"]), torch.empty_like(s["f"]), empty(s["w"], d), empty(s["b"], d), empty(s["wp"], d),
                    empty(s["bp"], d), None if s["gate"] is None else empty(level, *s["gate"].shape))
    if own:
        import paper_2501_14183_amd as vd
        kinds = {"none": vd.NORM_NONE, "layer": vd.NORM_LAYER, "rms": vd.NORM_RMS}
        s |= dict(vd=vd, ctx=context(vd), pre=kinds[c["pre"]], post=kinds[c["post"]])
        if c["path"] == "norm_bwd":
            s["ws"] = torch.empty(vd.vardrop_block_norm_workspace_bytes(B, n, d, 0 if s["gate"] is None else s["gate"].shape[0]),
                                  dtype=torch.uint8, device="cuda")
    return s


def prepare_tensors(c, g):
    first, rest = sizes(c)
    every, decayed = first + rest, sum(first)
    total = sum(every)
    scale = torch.empty(len(every), device="cuda").uniform_(-7.5, -3.5, generator=g).exp_()     # tensors differ in scale
    scale = torch.repeat_interleave(scale, torch.tensor(every, device="cuda"))
    flat = {"g": torch.randn(total, generator=g, device="cuda").mul_(scale).to(TYPES[c["grad"]])}
    if c["path"] == "clip":
        flat["out"] = torch.empty(total, dtype=TYPES[c["to"]], device="cuda")
    else:
        flat["p"] = torch.randn(total, generator=g, device="cuda").mul_(0.04)
        flat["m"] = torch.randn(total, generator=g, device="cuda").mul_(scale).mul_(0.2)
        flat["v"] = torch.rand(total, generator=g, device="cuda").add_(0.5).mul_(scale).mul_(scale)
        if c["to"] == "bf16":
            flat["w"] = flat["p"].to(torch.bfloat16)
    s = dict(c, flat=flat, decayed=decayed, norm=torch.empty(1, device="cuda"), step=200)
    if c["dev"]:
        s["step"] = torch.full((1,), 200, dtype=torch.int64, device="cuda")
        s["rate"] = torch.full((1,), RATE, dtype=torch.float32, device="cuda")
    if own:
        import paper_2501_14183_amd as vd
        part = {k: t.split(every) for k, t in flat.items()}
        s |= dict(vd=vd, ctx=context(vd))
        if c["path"] == "clip":
            s["list"] = vd.TensorList(s["ctx"], part["g"], clipped=part["out"])
        else:
            s["list"] = vd.TensorList(s["ctx"], part["g"], params=part["p"], exp_avg=part["m"], exp_avg_sq=part["v"],
                                      weights=part.get("w"), decay=[DECAY] * len(first) + [0.0] * len(rest))
    return s


contexts = []


def context(vd):
    """The one context of this process."""
    if not contexts:
        contexts.append(vd.Context(0))
    return contexts[0]


def run(s):
    return {"norm_fwd": run_norm_fwd, "norm_bwd": run_norm_bwd, "clip": run_clip, "adamw": run_adamw}[s["path"]](s)


def run_norm_fwd(s):
    if own:
        return s["vd"].vardrop_block_norm_fwd(s["ctx"], s["x"], s["f"], pre=s["pre"], w=s["w"], b=s["b"], post=s["post"], wp=s["wp"],
                                              bp=s["bp"], gate=s["gate"], alpha=s["alpha"], beta=s["beta"], eps=EPS_NORM, out=s["out"])
    return norm_forward(s)


def run_norm_bwd(s):
    if own:
        return s["vd"].vardrop_block_norm_bwd(s["ctx"], s["dr"], s["dh"], s["r"], s["f"], s["stats"], pre=s["pre"], w=s["w"],
                                              post=s["post"], wp=s["wp"], bp=s["bp"], gate=s["gate"], alpha=s["alpha"],
                                              beta=s["beta"], ws=s["ws"], out=s["out"])
    return norm_backward(s)


def run_clip(s):
    if own:
        norm_ = s["vd"].vardrop_grad_norm(s["ctx"], s["list"], out=s["norm"])
        s["vd"].vardrop_clip_grads(s["ctx"], s["list"], norm_, s["max_norm"])
        return norm_, s["flat"]["out"]
    g = s["flat"]["g"].float()
    norm_ = g.square().sum().sqrt().reshape(1)
    return norm_, s["flat"]["out"].copy_(g * clip_factor(norm_, s["max_norm"]))


def run_adamw(s):
    flat = s["flat"]
    if own:
        vd, norm_ = s["vd"], None
        if s["max_norm"] > 0:
            norm_ = vd.vardrop_grad_norm(s["ctx"], s["list"], out=s["norm"])
        if s["dev"]:
            vd.vardrop_adamw_dev(s["ctx"], s["list"], s["rate"], s["step"], beta1=BETA1, beta2=BETA2, eps=EPS_ADAM, norm=norm_,
                                 max_norm=s["max_norm"])
        else:
            s["step"] += 1
            vd.vardrop_adamw(s["ctx"], s["list"], RATE, s["step"], beta1=BETA1, beta2=BETA2, eps=EPS_ADAM, norm=norm_,
                             max_norm=s["max_norm"])
        return adamw_outputs(s, norm_)
    g, p, m, v, norm_ = flat["g"].float(), flat["p"], flat["m"], flat["v"], None
    if s["max_norm"] > 0:
        norm_ = g.square().sum().sqrt().reshape(1)
        g = g * clip_factor(norm_, s["max_norm"])
    s["step"] += 1
    rate = s["rate"] if s["dev"] else RATE
    m.copy_(BETA1 * m + (1 - BETA1) * g)
    v.copy_(BETA2 * v + (1 - BETA2) * g * g)
    step = m / (1 - BETA1 ** s["step"]) / ((v / (1 - BETA2 ** s["step"])).sqrt() + EPS_ADAM)
    p[:s["decayed"]].mul_(1 - rate * DECAY)
    p.sub_(rate * step)
    if "w" in flat:
        flat["w"].copy_(p)
    return adamw_outputs(s, norm_)


def adamw_outputs(s, norm_):
    flat = s["flat"]
    return {"norm": norm_, "p": flat["p"], "m": flat["m"], "v": flat["v"], "w": flat.get("w"), "step": s["step"]}


def clip_factor(norm_, max_norm):
    return (max_norm / (norm_ + EPS_CLIP)).clamp(max=1.0)


def statistics(kind, t):
    """Mean and reciprocal deviation of the rows of t (fp32), 0 and 1 where there is no norm, as columns."""
    if kind == "none":
        return torch.zeros_like(t[..., :1]), torch.ones_like(t[..., :1])
    mean = t.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(t[..., :1])
    return mean, ((t - mean).square().mean(-1, keepdim=True) + EPS_NORM).rsqrt()


def affine(t, w, b):
    t = t if w is None else t * w.float()
    return t if b is None else t + b.float()


def gate_rows(s):
    return None if s["gate"] is None else s["gate"].float().unsqueeze(1)     # [1 or B][1][d]


def norm_forward(s):
    x, f = s["x"].float(), s["f"].float()
    mean_p, rstd_p = statistics(s["post"], f)
    u = affine((f - mean_p) * rstd_p, s["wp"], s["bp"])
    u = u if s["gate"] is None else u * gate_rows(s)
    r = s["alpha"] * x + s["beta"] * u
    mean, rstd = statistics(s["pre"], r)
    h = affine((r - mean) * rstd, s["w"], s["b"])
    return r.to(s["x"].dtype), h.to(s["f"].dtype), torch.cat((mean_p, rstd_p, mean, rstd), -1).reshape(-1, 4)


def through_norm(kind, dt, hat, rstd):
    """Gradient of a norm's input rows, from that of the normalised rows."""
    if kind == "none":
        return dt
    dx = dt - hat * (dt * hat).mean(-1, keepdim=True)
    return rstd * (dx - dt.mean(-1, keepdim=True) if kind == "layer" else dx)


def norm_backward(s):
    B, n, d = s["x"].shape
    mean_p, rstd_p, mean, rstd = s["stats"].reshape(B, n, 4).split(1, -1)
    dh, f = s["dh"].float(), s["f"].float()
    hat = (s["r"].float() - mean) * rstd
    db, dw = dh.sum((0, 1)), (dh * hat).sum((0, 1))
    D = s["dr"].float() + through_norm(s["pre"], dh * s["w"].float(), hat, rstd)
    dx = s["alpha"] * D
    hat_p = (f - mean_p) * rstd_p
    du = s["beta"] * D
    dgate = None
    if s["gate"] is not None:
        dgate = du * affine(hat_p, s["wp"], s["bp"])
        dgate = dgate.sum((0, 1)).reshape(1, d) if s["gate"].shape[0] == 1 else dgate.sum(1)
        du = du * gate_rows(s)
    dwp = None if s["wp"] is None else (du * hat_p).sum((0, 1))
    dbp = None if s["bp"] is None else du.sum((0, 1))
    df = through_norm(s["post"], du if s["wp"] is None else du * s["wp"].float(), hat_p, rstd_p)
    return dx.to(s["x"].dtype), df.to(s["f"].dtype), dw, None if s["b"] is None else db, dwp, dbp, dgate


def work(c):
    wide = {"fp32": 4, "bf16": 2}
    if c["path"].startswith("norm"):
        rows, d = c["B"] * c["n"], c["d"]
        vectors = 1 + c["bias"] + (c["post"] != "none") * (1 + c["bias"]) + {"none": 0, "shared": 1, "window": c["B"]}[c["gate"]]
        if c["path"] == "norm_fwd":     # x, f -> r, h, statistics
            return {"bytes": rows * (2 * d * (wide[c["res"]] + wide[c["dtype"]]) + 16) + vectors * d * wide[c["dtype"]],
                    "flops": rows * d * 16}
        # dr, dh, r, f, statistics -> dx, df, gradients of the vectors
        return {"bytes": rows * (3 * d * (wide[c["res"]] + wide[c["dtype"]]) + 16) + vectors * d * (wide[c["dtype"]] + 4),
                "flops": rows * d * 30}
    total = sum(map(sum, sizes(c)))
    if c["path"] == "clip":
        return {"bytes": total * (wide[c["grad"]] + wide[c["to"]]), "flops": total * 3}
    return {"bytes": total * (wide[c["grad"]] + 24 + 2 * (c["to"] == "bf16")), "flops": total * (16 + 2 * (c["max_norm"] > 0))}


def exact(case, seed):
    """The outputs of run() from the definitions, in 64 bits."""
    s = prepare(case, seed)
    wide = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    return {"norm_fwd": exact_norm_fwd, "norm_bwd": exact_norm_bwd, "clip": exact_clip, "adamw": exact_adamw}[case["path"]](case, wide)


def exact_rows(kind, t):
    """(mean, 1 / deviation) of every row by moments about the mean, or about zero."""
    rows, d = t.reshape(-1, t.shape[-1]), t.shape[-1]
    at = rows.sum(1) / d * (kind == "layer")
    dev = ((rows - at[:, None]) ** 2).sum(1) / d
    one = torch.ones_like(at)
    return (at, one) if kind == "none" else (at, 1 / torch.sqrt(dev + EPS_NORM))


def exact_branch(case, s):
    """Factor and offset that turn a normalised row of f into the branch's share of r, for every token."""
    B, n, d = s["x"].shape
    one = torch.ones(d, dtype=torch.float64, device=s["x"].device)
    gate = one.expand(B, d) if s["gate"] is None else s["gate"].expand(B, d)
    wp = one if s["wp"] is None else s["wp"]
    bp = 0 * one if s["bp"] is None else s["bp"]
    return (case["beta"] * gate).repeat_interleave(n, 0), wp, bp


def exact_norm_fwd(case, s):
    B, n, d = s["x"].shape
    at_p, r_p = exact_rows(case["post"], s["f"])
    scale, wp, bp = exact_branch(case, s)
    f = s["f"].reshape(-1, d)
    r = case["alpha"] * s["x"].reshape(-1, d) + scale * (wp * (f - at_p[:, None]) * r_p[:, None] + bp)
    at, inv = exact_rows(case["pre"], r)
    h = s["w"] * (r - at[:, None]) * inv[:, None] + (0 if s["b"] is None else s["b"])
    return r.reshape(B, n, d), h.reshape(B, n, d), torch.stack((at_p, r_p, at, inv), 1)


def exact_norm_bwd(case, s):
    B, n, d = s["x"].shape
    at_p, r_p, at, inv = s["stats"].T

    def jacobian(kind, v, unit, k):
        """k (I - 1 1^T / d - unit unit^T / d) v, the ones only where the mean is taken out."""
        if kind == "none":
            return v
        along = (v * unit).sum(1) / d
        flat = v.sum(1) / d * (kind == "layer")
        return k[:, None] * (v - flat[:, None] - along[:, None] * unit)

    dh = s["dh"].reshape(-1, d)
    unit = inv[:, None] * (s["r"].reshape(-1, d) - at[:, None])
    D = s["dr"].reshape(-1, d) + jacobian(case["pre"], s["w"] * dh, unit, inv)
    scale, wp, bp = exact_branch(case, s)
    unit_p = r_p[:, None] * (s["f"].reshape(-1, d) - at_p[:, None])
    df = jacobian(case["post"], wp * scale * D, unit_p, r_p)
    dgate = None
    if s["gate"] is not None:
        dgate = (case["beta"] * D * (wp * unit_p + bp)).reshape(B, n, d).sum(1)
        dgate = dgate.sum(0, keepdim=True) if case["gate"] == "shared" else dgate
    return ((case["alpha"] * D).reshape(B, n, d), df.reshape(B, n, d), (dh * unit).sum(0), None if s["b"] is None else dh.sum(0),
            None if s["wp"] is None else (scale * D * unit_p).sum(0), None if s["bp"] is None else (scale * D).sum(0), dgate)


def exact_clip(case, s):
    g = s["flat"]["g"].double()
    length = torch.linalg.vector_norm(g)
    return length.reshape(1), g if length + EPS_CLIP <= case["max_norm"] else g / (length + EPS_CLIP) * case["max_norm"]


def exact_adamw(case, s):
    flat = {k: t.double() for k, t in s["flat"].items()}
    g, length, t = flat["g"], None, 201
    if case["max_norm"] > 0:
        length, g = exact_clip(case, s)
    m = flat["m"] + (g - flat["m"]) * (1 - BETA1)
    v = flat["v"] + (g * g - flat["v"]) * (1 - BETA2)
    shrink = torch.ones_like(g)
    shrink[:s["decayed"]] -= RATE * DECAY
    p = flat["p"] * shrink - RATE * (m / (1 - BETA1 ** t)) / (torch.sqrt(v) / (1 - BETA2 ** t) ** 0.5 + EPS_ADAM)
    return {"norm": length, "p": p, "m": m, "v": v, "w": p if "w" in flat else None, "step": 201}
