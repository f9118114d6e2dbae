"""Inputs of the tests of the feed-forward block's tiles, and the definitions in 64 bits on the tensors' own device (not a test module).

LARGE, LARGE_FP32, PARTS and LARGE_I8 are sizes with the tiles that the rules of the library choose for them; test_ffn_plan.py holds them to that.

Whole numbers.  x, W1, W2, dy of -1, 0, 1 and small biases, so few that |h| <= 127 and |dh| <= 256: x, h, act(h) = max(h, 0), dh and all sums
(below 2^24) are exact in every type and order, checkpoints too, and a result in bf16 is rounded once.  What the kernels give is
equal to the definition, bit for bit.

Single products (fp32).  Operands with one number in each row, or column, of the summed axis: every result is one product of numbers with 24-bit
mantissas, which shows every pair of their parts.  With u = 2^-24, x = hi + mid + lo exactly, |mid| <= 2^-8 |x|, |lo| <= 2^-16 |x|:
the pairs left out (mid lo, lo mid, lo lo) are 2 u of the product and 2^-32; of the six additions the last is off by 2 u at most (u if the
instruction rounds to nearest), the others by 2 u of what is below 2^-7: together less than 5 u.  A factor that has one part (a checkpoint's value) leaves none out: less than
3 u.  Two products in a row: 11 u.  A pair that is lost shows as 2^-17 = 128 u and less, depending on the numbers' bits: as more than the bound for
a good part of the elements.
GELU in fp32: 2 u (1 + |x|) by the fit (test_ffn_host.py evaluates it), and 1 for a further step of the exponential.

Dense fp32 products, by norm.  A sum of K products is 6 K / 16 additions of the matrix instruction; each off by 2 u of a partial sum, whose mean
square is half the whole's, signs by chance: u sqrt(6 K / 16 * 4 / 2) < u sqrt(K).  With 4 u for what is left out and GELU: (4 + sqrt(K1) + sqrt(K2)) u for two in a row.
"""
import torch

U = 2.0 ** -24
F64 = torch.float64

# (B, n, d, f): tiles (of kRowShapes for up and dh, of kShapes for down, of kShapes and slices for the gradients)
LARGE = {
    (1, 16001, 832, 1984): (2, 2, 2, 4),
    (1, 7001, 1984, 2112): (2, 2, 2, 1),
    (3, 10003, 448, 1600): (2, 2, 2, 6),
    (1, 50021, 192, 832): (2, 2, 1, 11),
    (1, 8111, 448, 1600): (2, 0, 2, 5),
    (1, 3001, 1088, 1088): (0, 0, 2, 3),
    (1, 6001, 832, 1088): (1, 1, 2, 4),
    (2, 10007, 64, 576): (1, 0, 0, 14),
}
# of kPartShapes
LARGE_FP32 = {
    (1, 6001, 450, 500): (1, 1, 1, 5),
    (1, 8001, 321, 449): (1, 1, 1, 6),
    (1, 600, 200, 66): (0, 0, 0, 5),
}
PARTS = {
    (1, 300, 100, 130): (0, 0, 0, 1),
    (1, 600, 200, 66): (0, 0, 0, 5),
    (1, 6001, 450, 500): (1, 1, 1, 5),
    (1, 8001, 321, 449): (1, 1, 1, 6),
}
# rows, K, N: tile of kRowShapes
LARGE_I8 = {(20011, 97, 721): 2, (27581, 512, 2047): 2, (20011, 512, 720): 2, (5003, 300, 1001): 1, (2999, 600, 33): 0}


def generator(*key, device="cuda"):
    return torch.Generator(device).manual_seed(sum((k + 1) * 7919 ** i for i, k in enumerate(key)) % (1 << 62))


# ---- the block in 64 bits
def cdf(t):
    return 0.5 * torch.special.erfc(t * -0.5 ** 0.5)


def act(kind, t):
    return torch.where(t < 0, 0.0, t) if kind == "relu" else t * cdf(t)


def slope(kind, t):
    return (t > 0).to(t.dtype) if kind == "relu" else cdf(t) + t * torch.exp(t * t / -2) / (2 * torch.pi) ** 0.5


def forward(t, kind):
    """(y, h) from tensors in 64 bits; biases may be missing."""
    h = t["x"] @ t["W1"]
    h = h if t["b1"] is None else h + t["b1"]
    y = act(kind, h) @ t["W2"]
    return (y if t["b2"] is None else y + t["b2"]), h


def backward(t, x, h, kind):
    dh = (t["dy"] @ t["W2"].t()) * slope(kind, h)
    return dict(dx=dh @ t["W1"].t(), dW1=x.t() @ dh, dW2=act(kind, h).t() @ t["dy"], db1=dh.sum(0), db2=t["dy"].sum(0))


def pack(rows):
    """Rows of finite numbers as an 8-bit checkpoint: (codes int8, exponent bytes uint8, the values they stand for)."""
    T, d = rows.shape
    codes, exps, values = [], [], []
    for at in range(0, d, 32):
        part = rows[:, at:at + 32].to(F64)
        most = part.abs().amax(1, keepdim=True)
        fraction, e = torch.frexp(most)                          # most = 2^e fraction, 1/2 <= fraction < 1
        e = (e.long() - 7 + (128 * fraction >= 127.5)).clamp(-126, 121)
        e = torch.where(most > 0, e, -126)
        step = ((e + 1023) << 52).view(F64)
        code = torch.round(part / step).clamp(-127, 127)
        codes.append(code.to(torch.int8))
        exps.append((e + 127).to(torch.uint8))
        values.append(code * step)
    return torch.cat(codes, 1), torch.cat(exps, 1), torch.cat(values, 1)


# ---- whole numbers
def whole_numbers(B, n, d, f, device="cuda"):
    T, g = B * n, generator(1, B, n, d, f, device=device)
    p = min(1.0, (150 * 9 / 4 / d) ** 0.5)

    def signs(*shape):
        return torch.randint(-1, 2, shape, generator=g, device=device).float() * (torch.rand(*shape, generator=g, device=device) < p)

    small = lambda k: torch.randint(-8, 9, (k,), generator=g, device=device).float()
    return dict(x=signs(T, d), W1=signs(d, f), b1=small(f), W2=signs(f, d), b2=small(d), dy=signs(T, d))


# ---- single products
def mantissas(g, *shape, signed=False):
    """Numbers of 1..2 (and -2..-1) with 24-bit mantissas."""
    t = 1 + torch.randint(0, 1 << 23, shape, generator=g, device=g.device).float() * 2.0 ** -23
    return t * (torch.randint(0, 2, shape, generator=g, device=g.device) * 2 - 1) if signed else t


def one_in_each(count, of, shift, device):
    """For each of `count` a place of `of`, in an order that visits all of them."""
    step = next(s for s in range(of // 3 + 1, 2 * of + 2) if torch.gcd(torch.tensor(s), torch.tensor(of)) == 1)
    return (torch.arange(count, device=device) * step + shift) % of


def sparse(rows, cols, row, col, values):
    t = torch.zeros(rows, cols, device=values.device)
    t[row, col] = values
    return t


def single_forward(T, d, f, shift, device="cuda"):
    """x has one number in each row, W2 one in each column: y[t][c] = x[t][at(t)] W1[at(t)][from(c)] W2[from(c)][c].  (ReLU, everything before it positive)"""
    g = generator(2, T, d, f, shift, device=device)
    t, c = torch.arange(T, device=device), torch.arange(d, device=device)
    return dict(x=sparse(T, d, t, one_in_each(T, d, shift, device), mantissas(g, T)), W1=mantissas(g, d, f), b1=None,
                W2=sparse(f, d, one_in_each(d, f, shift, device), c, mantissas(g, d, signed=True)), b2=None)


def single_backward(T, d, f, shift, device="cuda"):
    """dy has one number in each row, W1 one in each row, x one in each column, h is positive: dh, dx and dW1 are single products."""
    g = generator(3, T, d, f, shift, device=device)
    t, c = torch.arange(T, device=device), torch.arange(d, device=device)
    return dict(dy=sparse(T, d, t, one_in_each(T, d, shift, device), mantissas(g, T, signed=True)), W2=mantissas(g, f, d, signed=True),
                W1=sparse(d, f, c, one_in_each(d, f, shift, device), mantissas(g, d, signed=True)),
                x=sparse(T, d, one_in_each(d, T, shift, device), c, mantissas(g, d, signed=True)), h=mantissas(g, T, f))


def single_dW2(T, d, f, shift, device="cuda"):
    """dy has one number in each column: dW2 is made of single products of act(h)."""
    g = generator(4, T, d, f, shift, device=device)
    return dict(dy=sparse(T, d, one_in_each(d, T, shift, device), torch.arange(d, device=device), mantissas(g, d, signed=True)), W2=mantissas(g, f, d),
                W1=mantissas(g, d, f), x=mantissas(g, T, d), h=mantissas(g, T, f))


def dW2_bound(h, dy, want):
    return 3 * U * (1 + h.abs()).t() @ dy.abs() + 5 * U * want.abs()


def dense(T, d, f, device="cuda"):
    g = generator(5, T, d, f, device=device)
    normal = lambda *shape, scale=1.0: torch.randn(*shape, generator=g, device=device) * scale
    return dict(x=normal(T, d), W1=normal(d, f, scale=d ** -0.5), b1=normal(f, scale=0.1), W2=normal(f, d, scale=f ** -0.5), b2=normal(d, scale=0.1),
                dy=normal(T, d), h=normal(T, f))


def norm_bound(*K):
    return U * (4 + sum(k ** 0.5 for k in K))


def off(got, want):
    """Of the norm."""
    return float((got.to(F64) - want).norm() / want.norm())


def wide(t):
    return {k: v if v is None else v.to(F64) for k, v in t.items()}
