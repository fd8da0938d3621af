"""The orthogonalised update with the roundings that its kernel states, in 64-bit
arithmetic, and what a kernel's answer is held to.

Operands: X at 1024 times its size and A, C at 256 times, as one fp16 number or (`pairs`) as two, the second at 2^11
times its size.  A product's sum is a tensor core's, which adds 16 terms at a time to fp32 and truncates; pairs are
added up in fp32 every 64 terms.  The rest is fp32: C = b A + c A A of the stored A, X <- a X + C X of both parts of
X, with the diagonal of C beside a where operands are single.

`mistake` plants one.  `exact_sums` leaves the truncation of sums out: how far that moves the answer is what a
kernel's own order and width of sums may move it by, so the tolerance comes from the emulation alone."""
import torch

QUINTIC = (3.4445, -4.7750, 2.0315)
MISTAKES = ("zeros", "four steps", "b off by 1%", "a tile dropped", "a block stale", "bf16 operands", "no second parts",
            "mixed product dropped", "diagonal in the product", "a X in the product", "linear term of X's first part")


def make(rows, cols, dtype, seed=0, spread=True, device="cpu"):
    """A few strong directions and a small rest, or (not spread) independent elements."""
    g = torch.Generator(device=device).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device=device, generator=g)

    if not spread:
        return randn(rows, cols).to(dtype)
    k = min(rows, cols, 5)
    return ((randn(rows, k) * 0.5 ** torch.arange(k, device=device)) @ randn(k, cols) + 0.2 * randn(rows, cols)).to(dtype)


def f32(x):
    return x.float().double()


def toward_zero(x):
    """fp32 of a 64-bit value, truncated."""
    y = x.float()
    over = y.abs().double() > x.abs()
    return torch.where(over, torch.nextafter(y, torch.zeros_like(y)), y).double()


class Number:
    """Stored operands: first and second part, at `up` times their size."""

    def __init__(self, v, up, pairs, mistake):
        self.up = up
        first = v.float() * up
        self.first = (first.bfloat16() if mistake == "bf16 operands" else first.half()).double()
        second = ((first.double() - self.first) * 2048).float().half().double() / 2048
        self.second = second if pairs and mistake != "no second parts" else torch.zeros_like(second)

    def t(self):
        n = object.__new__(Number)
        n.up, n.first, n.second = self.up, self.first.t(), self.second.t()
        return n

    def value(self):
        return (self.first + self.second) / self.up


def product(x, y, pairs, exact_sums, mistake):
    """x y as the tensor cores sum it."""
    k = x.first.shape[1]
    down = 1.0 / (x.up * y.up)
    if exact_sums:
        v = x.first @ y.first
        if pairs:
            v = v + x.first @ y.second + (x.second @ y.first if mistake != "mixed product dropped" else 0)
        return f32(v * down)
    total = 0
    for k0 in range(0, k, 64 if pairs else k):
        ends = range(k0, min(k, k0 + 64) if pairs else k, 16)
        acc = 0
        if pairs:
            for i in ends:
                acc = toward_zero(acc + x.first[:, i:i + 16] @ y.second[i:i + 16])
                if mistake != "mixed product dropped":
                    acc = toward_zero(acc + x.second[:, i:i + 16] @ y.first[i:i + 16])
        for i in ends:
            acc = toward_zero(acc + x.first[:, i:i + 16] @ y.first[i:i + 16])
        total = f32(total + acc)
    return f32(total * down)


def emulate(u, pairs, steps=5, coefficients=QUINTIC, eps=1e-7, exact_sums=False, mistake=None):
    """X in 64 bits, before the result's rounding."""
    a, b, c = (float(torch.tensor(v)) for v in coefficients)
    flip = u.shape[0] > u.shape[1]
    x = u.double().t() if flip else u.double()
    x = f32(x / (x.square().sum().sqrt() + eps))
    if mistake == "zeros":
        return torch.zeros_like(u, dtype=torch.float64)
    if mistake == "b off by 1%":
        b = 1.01 * b
    if mistake == "four steps":
        steps -= 1
    how = pairs, exact_sums, mistake
    X = Number(x, 1024.0, True, mistake)
    last = None
    for step in range(steps):
        op = X if pairs else Number(X.first / X.up, 1024.0, False, mistake)
        A = Number(product(op, op.t(), *how), 256.0, pairs, mistake)
        C = f32(b * A.value() + c * product(A, A, *how))
        linear = torch.full((len(C), 1), a, dtype=torch.float64, device=u.device)
        if mistake == "a X in the product":
            C, linear = C + torch.diag(linear[:, 0]), torch.zeros_like(linear)
        elif not pairs and mistake != "diagonal in the product":
            linear = f32(linear + torch.diag(C)[:, None])
            C = C - torch.diag(torch.diag(C))
        kept = X.first / X.up if mistake == "linear term of X's first part" else X.value()
        new = f32(linear * kept + product(Number(C, 256.0, pairs, mistake), op, *how))
        if step == steps - 1 and mistake == "a tile dropped":
            new[128:256, 128:256] = 0
        if step == steps - 1 and mistake == "a block stale":
            new[:64, 64:128] = last[:64, 64:128]
        last = new
        X = Number(new, 1024.0, True, mistake)
    return last.t() if flip else last


def exact(u, steps=5, coefficients=QUINTIC, eps=1e-7):
    a, b, c = coefficients
    flip = u.shape[0] > u.shape[1]
    x = u.double().t() if flip else u.double()
    x = x / (x.norm() + eps)
    for _ in range(steps):
        A = x @ x.t()
        x = a * x + (b * A + c * A @ A) @ x
    return x.t() if flip else x


def blocks(x):
    """Squares of the norms of 64 x 64 blocks."""
    r, c = x.shape
    pad = torch.nn.functional.pad(x, (0, -c % 64, 0, -r % 64)).square()
    return pad.view(-(-r // 64), 64, -(-c // 64), 64).sum((1, 3))


class Held:
    """What an answer for `u` is held to, from two emulations, with truncated and with exact sums.

    Pairs: their roundings are as small as the sums' own, and an answer whose sums are of another order or width lies
    near the first emulation, by the measure of the second, whose sums are exact.  A tensor core cuts not the sum of
    16 products and the one before alone, which loses 2^-24 of it on average, but each of these 17 terms too, at the
    27th bit from the largest's first (outputs of six shapes agree with that): 17 * 2^-26 on average, all toward zero,
    17 / 4 of the former.  With the emulation's own loss that is 5.25 times as far from it as exact sums are: six times,
    and 3 * 2^-24 of the norm for fp32's order of the few other operations.  In each block within twice its share of
    that, for an uneven spread.
    Single operands: elements of A beside its diagonal are small against the terms that they are summed of, and an
    error of such a sum moves their fp16 rounding to the other side; after two steps the roundings of two emulations
    have nothing to do with each other, and what they share is their size.  Thousands of independent roundings add up
    to the same norm within a few hundredths: an answer is within 1.15 times the larger emulation's distance from 64
    bits, in each block within three times what it is there or its share."""

    def __init__(self, u, dtype, pairs, **how):
        self.dtype, self.pairs = dtype, pairs
        self.exact = exact(u, **how)
        self.near, other = (emulate(u, pairs, exact_sums=e, **how).to(dtype).double() for e in (False, True))
        self.offs = [float((x - self.exact).norm()) for x in (self.near, other)]
        share = blocks(torch.ones_like(other)) / other.numel()
        if pairs:
            self.room = 6 * float((other - self.near).norm()) + 3 * 2.0 ** -24 * float(other.norm())
            self.block_room = (2 * self.room) ** 2 * share
        else:
            self.room = 1.15 * max(self.offs)
            self.block_room = 9 * torch.maximum(torch.maximum(blocks(self.near - self.exact), blocks(other - self.exact)), self.room ** 2 * share)

    def why_not(self, got):
        """None, or what is wrong with an answer."""
        got = got.to(self.dtype).double()
        d = got - (self.near if self.pairs else self.exact)
        if not float(d.norm()) <= self.room:
            return f"{float(d.norm()):.3g} off, {self.room:.3g} allowed"
        if not bool((blocks(d) <= self.block_room).all()):
            return f"a block is {float((blocks(d) / self.block_room).max().sqrt()):.3g} times as far off as allowed"
        return None
