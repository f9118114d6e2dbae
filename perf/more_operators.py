"""Performance cases of the other half of an encoder layer, the feed-forward block, and of the two ways in which it is held in 8 bits:
checkpoints of activations for its backward pass, and 8-bit products for a model that answers.

A case is one of five calls ("path"):

  checkpoint  an activation is put away in 8 bits (blocks of 32 channels, one power of two for each) and fetched again
  ffn_fwd     y = act(x W1 + b1) W2 + b2 of a model that answers
  ffn_train   the same in training, x and h = x W1 + b1 kept in 8 bits, and its gradients from them
  ffn_bwd     the gradients alone, from checkpoints in hand
  linear_i8   y = act(x W + b) from 8-bit integers: a scale for each token and for each output channel

act is ReLU or GELU (x Phi(x)), or nothing for linear_i8.  Gradients come in the type of the weights.
"""
import torch

own = False
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32
MOST_CHECKPOINT, MOST_BF16, MOST_FP32, MOST_I8 = 32 * 862 * 1024, 8 * 8192 * 768 * 1536, 2 * 1001 * 512 * 1024, 8 * 8192 * 768 * 768


def listed():
    return [
        # The output of a layer's attention, all 862 variates of Traffic, put away until the backward pass.
        checkpoint("checkpoint_traffic_dense", 32, 862, 512, "bf16"),
        # An fp32 residual stream of an odd width: the last block of a row is short, rows begin anywhere.
        checkpoint("checkpoint_odd_fp32", 7, 321, 321, "fp32"),
        # The smallest workload of the repository, 10 of 32 variates kept.  Launches count.
        ffn("ffn_fwd_tiny_fp32", "ffn_fwd", 4, 10, 64, 128, "fp32", "relu"),
        # Forecasts for all 862 variates of Traffic.
        ffn("ffn_fwd_traffic_dense", "ffn_fwd", 32, 862, 512, 2048, "bf16", "gelu"),
        # The everyday training shape: kept tokens of Traffic, inner width as the model's.
        ffn("ffn_train_traffic", "ffn_train", 32, 87, 512, 512, "bf16", "relu"),
        # The largest: all 8192 variates of 8 windows at width 768.
        ffn("ffn_train_stress_dense", "ffn_train", 8, 8192, 768, 1536, "bf16", "gelu"),
        # All variates of Electricity, widths that no large tile divides.
        ffn("ffn_bwd_electricity_dense", "ffn_bwd", 7, 321, 320, 832, "bf16", "gelu"),
        # fp32 weights of odd widths.
        ffn("ffn_bwd_odd_fp32", "ffn_bwd", 3, 333, 321, 449, "fp32", "gelu"),
        # One token.
        linear("linear_i8_token", 1, 512, 512, "bf16", "none"),
        # Windows of 97 samples of all variates of Electricity to 321 channels, in and out in fp32: nothing is a whole tile.
        linear("linear_i8_odd", 7 * 321, 97, 321, "fp32", "none"),
        # The head of a model: one window of Traffic, 720 steps ahead.
        linear("linear_i8_head", 862, 512, 720, "bf16", "none"),
        # The first product of a feed-forward block over 32 windows of Traffic.
        linear("linear_i8_traffic_dense", 32 * 862, 512, 2048, "bf16", "gelu"),
    ]


def checkpoint(name, B, n, d, dtype):
    return dict(name=name, path="checkpoint", B=B, n=n, d=d, dtype=dtype)


def ffn(name, path, B, n, d, f, dtype, act, bias=True):
    return dict(name=name, path=path, B=B, n=n, d=d, f=f, dtype=dtype, act=act, bias=bias)


def linear(name, T, K, N, dtype, act, bias=True):
    return dict(name=name, path="linear_i8", T=T, K=K, N=N, dtype=dtype, act=act, bias=bias)


def spread(rng, lo, hi):
    """A whole number of lo..hi, evenly over its logarithm."""
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random() + rng.random())))


def draw(rng):
    path = rng.choice(("checkpoint", "ffn_fwd", "ffn_train", "ffn_bwd", "linear_i8"))
    if path == "checkpoint":
        d = rng.choice((64, 128, 320, 512, 768)) if rng.random() < 0.5 else spread(rng, 16, 2048)
        B = spread(rng, 1, 32)
        c = checkpoint("", B, spread(rng, 1, min(8192, MOST_CHECKPOINT // (B * d))), d, rng.choice(("fp32", "bf16")))
    elif path == "linear_i8":
        K, N = spread(rng, 16, 2048), spread(rng, 8, 2048)
        if rng.random() < 0.5:
            K, N = -(-K // 64) * 64, -(-N // 32) * 32
        c = linear("", spread(rng, 1, min(8 * 8192, MOST_I8 // (K * N))), K, N, rng.choice(("fp32", "bf16", "bf16")),
                   rng.choice(("none", "relu", "gelu")), rng.random() < 0.7)
    else:
        dtype = "fp32" if path != "ffn_train" and rng.random() < 0.3 else "bf16"
        if dtype == "fp32":
            d, f, most = spread(rng, 16, 512), spread(rng, 16, 1024), MOST_FP32
        else:
            d, f, most = 64 * spread(rng, 1, 16), 64 * spread(rng, 1, 32), MOST_BF16
        B = spread(rng, 1, 32)
        c = ffn("", path, B, spread(rng, 1, min(8192, most // (B * d * f))), d, f, dtype, rng.choice(("relu", "gelu")), rng.random() < 0.7)
    del c["name"]
    return c


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, at=0.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(scale).add_(at)

    def tokens(*shape):
        """Activations: channels differ in level and scale, a few by far."""
        loud = 0.4 + normal(shape[-1]).square_() * 0.4
        return normal(*shape).mul_(loud).add_(normal(shape[-1], scale=0.3))

    s = prepare_linear(case, normal, tokens) if case["path"] == "linear_i8" else prepare_block(case, normal, tokens)
    if own:
        import paper_2501_14183_amd as vd
        kinds = {"none": vd.ACT_NONE, "relu": vd.ACT_RELU, "gelu": vd.ACT_GELU}
        s |= dict(vd=vd, ctx=context(vd), kind=kinds[case.get("act", "none")])
        own_buffers(s)
    return s


def prepare_linear(c, normal, tokens):
    dt = TYPES[c["dtype"]]
    s = dict(c, x=tokens(c["T"], c["K"]).to(dt), W=normal(c["K"], c["N"], scale=c["K"] ** -0.5).to(dt),
             b=normal(c["N"], scale=0.1).to(dt) if c["bias"] else None)
    if not own:
        s["codes"], s["scale"] = integers(s["W"].float().t())
    return s


def prepare_block(c, normal, tokens):
    B, n, d, dt = c["B"], c["n"], c["d"], TYPES[c["dtype"]]
    s = dict(c, x=tokens(B, n, d).to(dt))
    if c["path"] == "checkpoint":
        return s
    f = c["f"]
    s |= dict(W1=normal(d, f, scale=d ** -0.5).to(dt), b1=normal(f, scale=0.1).to(dt) if c["bias"] else None,
              W2=normal(f, d, scale=f ** -0.5).to(dt), b2=normal(d, scale=0.1).to(dt) if c["bias"] else None)
    if c["path"] != "ffn_fwd":
        s["dy"] = normal(B, n, d, scale=0.01).to(dt)
    if c["path"] == "ffn_bwd":
        s["h"] = tokens(B, n, f).to(dt)
        if not own:
            s["kept"] = pack(s["x"].float()), pack(s["h"].float())
    return s


contexts = []


def context(vd):
    """The one context of this process."""
    if not contexts:
        contexts.append(vd.Context(0))
    return contexts[0]


def own_buffers(s):
    """What a program that makes the call again and again keeps: results, checkpoints, workspaces, weights in 8 bits."""
    vd, ctx, x = s["vd"], s["ctx"], s["x"]

    def room(nbytes):
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda")

    if s["path"] == "linear_i8":
        s["codes"], s["scale"] = vd.vardrop_quantize_weight(ctx, s["W"])
        s["y"] = torch.empty(s["T"], s["N"], dtype=x.dtype, device="cuda")
        s["ws"] = room(vd.vardrop_linear_i8_workspace_bytes(s["T"], s["K"], s["N"]))
        return
    B, n, d = x.shape
    if s["path"] == "checkpoint":
        s["saved"], s["back"] = room(vd.vardrop_pack8_bytes(B, n, d)), torch.empty_like(x)
        return
    f = s["f"]
    s["y"] = torch.empty_like(x)
    s["ws"] = room(vd.vardrop_ffn_workspace_bytes(B, n, d, f, x.dtype))
    if s["path"] != "ffn_fwd":
        s["saved"] = room(vd.vardrop_ffn_saved_bytes(B, n, d, f))
        vector = torch.empty_like if s["bias"] else lambda t: None
        s["grads"] = (torch.empty_like(x), torch.empty_like(s["W1"]), torch.empty_like(s["W2"]), vector(s["b1"]), vector(s["b2"]))
    if s["path"] == "ffn_bwd":
        first = vd.vardrop_pack8_bytes(B, n, d)
        vd.vardrop_pack8(ctx, x, out=s["saved"][:first])
        vd.vardrop_pack8(ctx, s["h"], out=s["saved"][first:])


def run(s):
    return {"checkpoint": run_checkpoint, "ffn_fwd": run_ffn_fwd, "ffn_train": run_ffn_train, "ffn_bwd": run_ffn_bwd,
            "linear_i8": run_linear_i8}[s["path"]](s)


def run_checkpoint(s):
    if own:
        s["vd"].vardrop_pack8(s["ctx"], s["x"], out=s["saved"])
        return s["vd"].vardrop_unpack8(s["ctx"], s["saved"], out=s["back"])
    return unpack(*pack(s["x"].float())).to(s["x"].dtype)


def run_ffn_fwd(s):
    if own:
        return s["vd"].vardrop_ffn_fwd(s["ctx"], s["x"], s["W1"], s["W2"], s["b1"], s["b2"], act=s["kind"], train=False, ws=s["ws"],
                                       out=s["y"])[0]
    return block(s)[0].to(s["x"].dtype)


def run_ffn_train(s):
    if own:
        y, _ = s["vd"].vardrop_ffn_fwd(s["ctx"], s["x"], s["W1"], s["W2"], s["b1"], s["b2"], act=s["kind"], saved=s["saved"], ws=s["ws"],
                                       out=s["y"])
        return y, own_gradients(s)
    y, h = block(s)
    return y.to(s["x"].dtype), block_gradients(s, pack(s["x"].float()), pack(h))


def run_ffn_bwd(s):
    return own_gradients(s) if own else block_gradients(s, *s["kept"])


def own_gradients(s):
    return s["vd"].vardrop_ffn_bwd(s["ctx"], s["dy"], s["W1"], s["W2"], s["saved"], act=s["kind"], ws=s["ws"], out=s["grads"])


def run_linear_i8(s):
    if own:
        return s["vd"].vardrop_linear_i8(s["ctx"], s["x"], s["codes"], s["scale"], s["b"], act=s["kind"], ws=s["ws"], out=s["y"])
    q, scale = integers(s["x"].float())
    y = (q.float() @ s["codes"].float().t()) * scale * s["scale"].t()
    return activation(s["act"], y if s["b"] is None else y + s["b"].float()).to(s["x"].dtype)


def integers(rows):
    """Rows as integers of -127..127 (nearest, ties to even) times a scale for each: (codes, scale as a column)."""
    most = rows.abs().amax(-1, keepdim=True)
    some = most >= 2.0 ** -100
    up = torch.where(some, 127.0 / most, torch.zeros_like(most))
    return (rows * up).round().to(torch.int8), torch.where(some, most / 127.0, torch.zeros_like(most))


def power(e):
    """2^e in fp32 for whole e of -126..127."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def pack(t):
    """Rows in blocks of 32 channels: the smallest power of two of which the block's largest value is at most 127, and integers."""
    d = t.shape[-1]
    t = torch.nn.functional.pad(t, (0, -d % BLOCK)).unflatten(-1, (-1, BLOCK))
    bits = t.abs().amax(-1, keepdim=True).view(torch.int32)
    e = (((bits + 0x10000) >> 23) - 127 - 6).clamp(-126, 121)
    return (t * power(-e)).round().clamp(-127, 127).to(torch.int8), e.to(torch.int8), d


def unpack(q, e, d):
    return (q.float() * power(e.to(torch.int32))).flatten(-2)[..., :d]


def cdf(t):
    return 0.5 * (1.0 + torch.erf(t * 0.5 ** 0.5))


def activation(kind, t):
    return t if kind == "none" else t.clamp(min=0.0) if kind == "relu" else t * cdf(t)


def slope(kind, t):
    return (t > 0).float() if kind == "relu" else cdf(t) + t * torch.exp(-0.5 * t * t) * (0.5 / torch.pi) ** 0.5


def block(s):
    """(y, h), both in fp32."""
    h = s["x"].float() @ s["W1"].float()
    h = h if s["b1"] is None else h + s["b1"].float()
    y = activation(s["act"], h) @ s["W2"].float()
    return (y if s["b2"] is None else y + s["b2"].float()), h


def block_gradients(s, kept_x, kept_h):
    x, h, dy = unpack(*kept_x).flatten(0, 1), unpack(*kept_h).flatten(0, 1), s["dy"].float().flatten(0, 1)
    dt = s["x"].dtype
    dh = (dy @ s["W2"].float().t()) * slope(s["act"], h)
    dx = (dh @ s["W1"].float().t()).reshape(s["x"].shape)
    dW1, dW2 = x.t() @ dh, activation(s["act"], h).t() @ dy
    db = (dh.sum(0).to(dt), dy.sum(0).to(dt)) if s["bias"] else (None, None)
    return dx.to(dt), dW1.to(dt), dW2.to(dt), *db


def work(c):
    wide = {"fp32": 4, "bf16": 2}[c["dtype"]]
    if c["path"] == "linear_i8":
        T, K, N = c["T"], c["K"], c["N"]
        return {"bytes": T * (K + N) * wide + K * N + 4 * N + N * wide * c["bias"], "flops": 2 * T * K * N}
    T, d = c["B"] * c["n"], c["d"]
    kept = 33 / 32
    if c["path"] == "checkpoint":
        return {"bytes": T * d * (2 * wide + 2 * kept), "flops": 6 * T * d}
    f = c["f"]
    weights = (2 * d * f + (d + f) * c["bias"]) * wide
    return {"ffn_fwd": {"bytes": 2 * T * d * wide + weights, "flops": 4 * T * d * f},
            "ffn_train": {"bytes": 4 * T * d * wide + 2 * T * (d + f) * kept + 2 * weights, "flops": 12 * T * d * f},
            "ffn_bwd": {"bytes": 2 * T * d * wide + T * (d + f) * kept + 2 * weights, "flops": 8 * T * d * f}}[c["path"]]


def exact(case, seed):
    """The outputs of run() from the definitions, in 64 bits."""
    s = prepare(case, seed)
    wide = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    if case["path"] == "linear_i8":
        return exact_linear(case, s, wide)
    if case["path"] == "checkpoint":
        return exact_kept(wide["x"])
    x, W1, W2 = wide["x"].reshape(-1, case["d"]), wide["W1"], wide["W2"]
    zero = torch.zeros(1, dtype=torch.float64, device=x.device)
    if case["path"] == "ffn_bwd":
        return exact_gradients(case, wide, x, wide["h"].reshape(-1, case["f"]))
    h = torch.addmm(zero if s["b1"] is None else wide["b1"], x, W1)
    y = torch.addmm(zero if s["b2"] is None else wide["b2"], exact_activation(case["act"], h)[0], W2).reshape(s["x"].shape)
    return y if case["path"] == "ffn_fwd" else (y, exact_gradients(case, wide, x, h))


def exact_kept(t):
    """What an 8-bit checkpoint of t stands for: a block's step is a power of two, a value the nearest multiple of it."""
    rows = t.reshape(-1, t.shape[-1])
    out = torch.empty_like(rows)
    for at in range(0, rows.shape[1], BLOCK):
        part = rows[:, at:at + BLOCK]
        fraction, e = torch.frexp(part.abs().max(1, keepdim=True).values)       # 2^e fraction, 1/2 <= fraction < 1
        e = e.long() - 7 + (128 * fraction >= 127.5)
        step = ((e + 1023) << 52).view(torch.float64)                           # (a power function would be a unit off now and then)
        out[:, at:at + BLOCK] = torch.round(part / step) * step
    return out.reshape(t.shape)


def exact_activation(kind, h):
    """Value and derivative."""
    if kind == "none":
        return h, torch.ones_like(h)
    if kind == "relu":
        return torch.where(h > 0, h, 0.0), (h > 0).double()
    below = 0.5 * torch.special.erfc(h * -0.5 ** 0.5)
    return h * below, below + h * torch.exp(h * h / -2) / (2 * torch.pi) ** 0.5


def exact_gradients(case, s, x, h):
    x, h, dy = exact_kept(x), exact_kept(h), s["dy"].reshape(-1, case["d"])
    a, rise = exact_activation(case["act"], h)
    dh = torch.mm(dy, s["W2"].T) * rise
    both = (dh.sum(0), dy.sum(0)) if case["bias"] else (None, None)
    return torch.mm(dh, s["W1"].T).reshape(s["dy"].shape), torch.mm(x.T, dh), torch.mm(a.T, dy), *both


def exact_linear(case, s, wide):
    def whole(t):
        """Codes and scales of the rows of t: the scale and its reciprocal are fp32 numbers by definition."""
        top = t.float().abs().max(1).values
        return torch.round((t.float() * (127 / top)[:, None])).double(), (top / 127).double()

    q, scale = whole(s["x"])
    w, channel = whole(s["W"].T)
    y = torch.mm(q, w.T) * torch.outer(scale, channel)
    return exact_activation(case["act"], y if s["b"] is None else y + wide["b"])[0]
