"""Cases that time the operators around the attention of a device's transformer
blocks: the embedding of its tokens with the gradient of the table, the root-mean-
square norm of a residual's addition with its gradient and its 8-bit form for
uploads, and the orthogonalised update of its weight matrices.

``run`` computes a case in plain torch operations (``own`` false) or through the
package's entry points (``own`` true).  ``exact`` gives the same outputs from the
definitions in 64 bits.

Definitions.
    Embedding: out_t = scale * table[id_t], zeros where id_t is outside 0 .. vocab - 1 (padding);
    its gradient dtable[v] = scale * sum of dout_t over the t with id_t = v.
    Norm: s = x + residual, rounded to the tensors' type; r = (mean_c s_c^2 + eps)^(-1/2); y_c = s_c r w_c.
    Gradient, for dy and the gradient ds that reaches s by the residual stream:
    dx = r (w dy - s r^2 mean_c(w_c dy_c s_c)) + ds (also the residual's), dw = sum over rows of dy s r.
    8-bit form of y: each 32 columns share the smallest power of two (2^-127 .. 2^127) with max|y| / 2^e <= 448;
    y / 2^e is rounded to a float of 4 exponent and 3 mantissa bits.
    Orthogonalised update of a matrix G with m <= n (or of its transpose): X = G / (|G|_F + eps), then `steps` times
    A = X X^T, X <- a X + (b A + c A A) X.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
EPS = 1e-6
STEPS, COEFFICIENTS, NORM_EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


def _embedding(name, direction, table, dtype, tokens, vocab, width, padded=False):
    """One embedding case.  table, dtype: types of the table (and its gradient) and of the activations; direction
    "forward", or "train" with the gradient; padded: a quarter of the tokens is padding."""
    return {"name": name, "op": "embedding", "direction": direction, "table": table, "dtype": dtype, "tokens": tokens,
            "vocab": vocab, "width": width, "padded": padded}


def _norm(name, direction, dtype, rows, cols, weight="", residual=True):
    """One norm case.  direction "forward", "train" (with the gradient) or "upload" (the 8-bit form and back);
    weight: the weight's type where it is not the activations'."""
    return {"name": name, "op": "norm", "direction": direction, "dtype": dtype, "weight": weight or dtype, "rows": rows,
            "cols": cols, "residual": residual}


def _orthogonalize(name, dtype, shapes):
    """Updates of several weight matrices, "rowsxcols" each, separated by commas."""
    return {"name": name, "op": "orthogonalize", "dtype": dtype, "shapes": shapes}


def listed():
    return [
        # one new token of each of 32 sequences: nothing but latency
        _embedding("embedding 32 tokens", "forward", "f32", "bf16", 32, 30522, 512),
        # the transformer workload's batch, 32 sequences padded to 128, fp32 parameters and bf16 activations: the
        # gradient's table is far larger than the batch
        _embedding("embedding 32x128", "train", "f32", "bf16", 4096, 30522, 512, padded=True),
        # few tokens to choose from, each many times; odd width, single precision
        _embedding("embedding f32 5000x777", "train", "f32", "f32", 5000, 1000, 777),
        # a large batch with a large table
        _embedding("embedding 65536x2048", "train", "bf16", "bf16", 65536, 100000, 2048),
        # one token of each of 32 sequences
        _norm("norm 32x512", "forward", "bf16", 32, 512),
        # the transformer workload's batch, fp32 weights
        _norm("norm 4096x512", "train", "bf16", 4096, 512, weight="f32"),
        # odd sizes in single precision
        _norm("norm f32 1000x777", "train", "f32", 1000, 777),
        # a large batch of wide activations
        _norm("norm 32768x4096", "train", "bf16", 32768, 4096),
        # split-point activations of a large batch, uploaded in 8 bits
        _norm("norm upload 16384x2048", "upload", "bf16", 16384, 2048),
        # one small matrix
        _orthogonalize("orthogonalize f32 200x96", "f32", "200x96"),
        # the matrices of two blocks of width 512, fp32 gradients
        _orthogonalize("orthogonalize blocks", "f32", ",".join(["1536x512", "512x512", "2048x512", "512x2048"] * 2)),
        # one large matrix, bf16 gradient
        _orthogonalize("orthogonalize 4096x4096", "bf16", "4096x4096"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _products(shapes):
    """Multiplications and additions of the updates of these matrices; A and A A are symmetric, and one half of each
    is enough."""
    total = 0
    for r, c in shapes:
        m, n = min(r, c), max(r, c)
        total += STEPS * (3 * m * m * n + m * m * m)
    return total


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def draw(rng):
    op = rng.choice(["embedding", "norm", "norm", "orthogonalize"])
    if op == "embedding":
        table, dtype = rng.choice([("f32", "bf16"), ("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
        e = BYTES[table]
        width = _log_int(rng, 8, 2048)
        if rng.random() < 0.5:
            width = max(8, width // 8 * 8)
        room = 400_000_000 // (width * e)
        c = _embedding("", rng.choice(["forward", "train", "train"]), table, dtype,
                       _log_int(rng, 1, min(65536, 65536 * 2048 * 2 // (width * BYTES[dtype]))), _log_int(rng, 100, min(100000, room)),
                       width, padded=rng.random() < 0.3)
    elif op == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        cols = _log_int(rng, 8, 8192)
        if rng.random() < 0.5:
            cols = max(8, cols // 8 * 8)
        rows = _log_int(rng, 1, min(65536, 32768 * 4096 * 2 // (cols * BYTES[dtype])))
        c = _norm("", rng.choice(["forward", "train", "train", "upload"]), dtype, rows, cols,
                  weight=rng.choice([dtype, "f32"]), residual=rng.random() < 0.8)
    else:
        dtype = rng.choice(["bf16", "f32"])
        room = _products([(4096, 4096)]) / (3 if dtype == "f32" else 1)
        shapes = []
        for _ in range(rng.randint(1, 8)):
            r, k = _log_int(rng, 8, 4096), _log_int(rng, 8, 4096)
            if rng.random() < 0.5:
                r, k = max(8, r // 8 * 8), max(8, k // 8 * 8)
            if _products(shapes + [(r, k)]) <= room:
                shapes.append((r, k))
        shapes = shapes or [(r // 2, k // 2)]
        c = _orthogonalize("", dtype, ",".join("%dx%d" % s for s in shapes))
    del c["name"]
    return c


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g, dtype=torch.float32)

    s = dict(case)
    t = TYPES[case["dtype"]]
    if case["op"] == "embedding":
        T, V, D = case["tokens"], case["vocab"], case["width"]
        # tokens of a text: the n-th most frequent one comes about 1 / n as often as the first
        u = torch.rand(T, device="cuda", generator=g, dtype=torch.float64)
        ids = (torch.pow(float(V + 1), u).long() - 1).clamp_(0, V - 1).to(torch.int32)
        if case["padded"]:
            ids[torch.rand(T, device="cuda", generator=g) < 0.25] = -1
        s["ids"], s["weights"], s["scale"] = ids, randn(V, D).to(TYPES[case["table"]]), math.sqrt(D)
        s["dout"] = (0.01 * randn(T, D)).to(t) if case["direction"] == "train" else None
        return s
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        # a few channels of transformer activations are far larger than the others
        channel = torch.exp(0.7 * randn(cols))
        s["x"] = (randn(rows, cols) * channel).to(t)
        s["residual"] = (3 * randn(rows, cols) * channel).to(t) if case["residual"] else None
        s["w"] = (1 + 0.2 * randn(cols)).to(TYPES[case["weight"]])
        if case["direction"] == "train":
            s["dy"], s["ds"] = randn(rows, cols).to(t), randn(rows, cols).to(t) if case["residual"] else None
        return s
    # gradients of weight matrices: a few strong directions and a small rest
    s["updates"] = []
    for r, c in _shapes(case):
        k = min(r, c, 8)
        s["updates"].append((1e-3 * (randn(r, k) * 0.6 ** torch.arange(k, device="cuda")) @ randn(k, c) + 2e-4 * randn(r, c)).to(t))
    return s


# ------------------------------------------------------------------ plain forms
def _plain_embedding(s):
    T, V, D = s["tokens"], s["vocab"], s["width"]
    ids = s["ids"].long()
    fine = ((ids >= 0) & (ids < V))[:, None]
    at = ids.clamp(0, V - 1)
    out = {"out": torch.where(fine, s["weights"][at].float() * s["scale"], 0.0).to(TYPES[s["dtype"]])}
    if s["direction"] == "train":
        grad = torch.zeros(V, D, device=ids.device)
        grad.index_add_(0, at, torch.where(fine, s["dout"].float(), 0.0))
        out["dtable"] = (grad * s["scale"]).to(TYPES[s["table"]])
    return out


def _plain_sum(s):
    """(s in the tensors' type, the same in 32 bits, r)."""
    x = s["x"]
    total = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    z = total.float()
    return total, z, torch.rsqrt(z.square().mean(1, keepdim=True) + EPS)


def _plain_norm(s):
    t = TYPES[s["dtype"]]
    total, z, r = _plain_sum(s)
    w = s["w"].float()
    y = z * r * w
    if s["direction"] == "upload":
        return {"s": total, "y": _plain_eight_bits(y)}
    out = {"s": total, "y": y.to(t), "r": r[:, 0]}
    if s["direction"] == "train":
        dy = s["dy"].float()
        g = dy * w
        dx = r * (g - z * r.square() * (g * z).mean(1, keepdim=True))
        if s["ds"] is not None:
            dx = dx + s["ds"].float()
        out["dx"] = dx.to(t)
        out["dw"] = (dy * z * r).sum(0).to(s["w"].dtype)
    return out


def _plain_eight_bits(y):
    """The values, in bf16, that the 8-bit form of y stands for (both the scales and the values fit)."""
    rows, cols = y.shape
    n = -(-cols // 32)
    z = torch.nn.functional.pad(y, (0, 32 * n - cols)).view(rows, n, 32)
    top = z.abs().amax(2, keepdim=True)
    m, e = torch.frexp(top)                     # top = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(top > 0, e - 9 + (m > 0.875), -127).clamp(-127, 127)
    z = torch.ldexp(z, -e)
    # steps of 2^-3 of the leading power of two, and of 2^-9 below 2^-6; ties to even
    step = torch.ldexp(torch.ones_like(z), (torch.frexp(z)[1] - 1).clamp(min=-6) - 3)
    z = torch.ldexp(torch.round(z / step) * step, e)
    return z.view(rows, 32 * n)[:, :cols].to(torch.bfloat16)


def _plain_orthogonalize(u):
    a, b, c = COEFFICIENTS
    x = u.float()
    if u.shape[0] > u.shape[1]:
        x = x.t()
    x = x / (x.square().sum().sqrt() + NORM_EPS)
    for _ in range(STEPS):
        A = torch.matmul(x, x.t())
        x = a * x + torch.matmul(b * A + c * torch.matmul(A, A), x)
    return (x.t() if u.shape[0] > u.shape[1] else x).to(u.dtype)


def run(s):
    if not own:
        if s["op"] == "orthogonalize":
            return [_plain_orthogonalize(u) for u in s["updates"]]
        return _plain_embedding(s) if s["op"] == "embedding" else _plain_norm(s)
    from paper_2504_13850_gb300 import api

    if s["op"] == "orthogonalize":
        return api.orthogonalize(s["updates"], steps=STEPS, coefficients=COEFFICIENTS, eps=NORM_EPS)
    if s["op"] == "embedding":
        out = {"out": api.embedding(s["ids"], s["weights"], scale=s["scale"], dtype=TYPES[s["dtype"]])}
        if s["direction"] == "train":
            out["dtable"] = api.embedding_grad(s["dout"], s["ids"], s["vocab"], scale=s["scale"], dtype=TYPES[s["table"]])
        return out
    if s["direction"] == "upload":
        q, scales, total = api.rms_norm_8bit(s["x"], s["residual"], s["w"], eps=EPS)
        return {"s": total, "y": api.decode_8bit(q, scales, dtype=torch.bfloat16)}
    y, total, r = api.rms_norm(s["x"], s["residual"], s["w"], eps=EPS)
    out = {"s": total, "y": y, "r": r}
    if s["direction"] == "train":
        out["dx"], out["dw"] = api.rms_norm_grad(s["dy"], s["ds"], total, s["w"], r)
    return out


def _used_rows(case):
    """How many rows of the table a batch uses, on average."""
    T, V = case["tokens"] * (0.75 if case["padded"] else 1.0), case["vocab"]
    n = np.arange(1, V + 1, dtype=np.float64)
    p = np.log1p(1 / n) / math.log(V + 1)
    return float(-np.expm1(T * np.log1p(-p)).sum())


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "embedding":
        T, V, D, f = case["tokens"], case["vocab"], case["width"], BYTES[case["table"]]
        count, flops = 4 * T + _used_rows(case) * D * f + T * D * e, T * D
        if case["direction"] == "train":        # reads dout, writes the whole table's gradient
            count, flops = count + T * D * e * (0.75 if case["padded"] else 1.0) + V * D * f, 2 * flops
        return {"bytes": count, "flops": flops}
    if case["op"] == "norm":
        n, r = case["rows"] * case["cols"], 1 if case["residual"] else 0
        if case["direction"] == "upload":       # x, residual; s, the 8-bit form and its scales; the same again and y
            return {"bytes": n * e * (1 + 2 * r) + 2 * (n + n / 32) + 2 * n, "flops": 8 * n}
        count = n * e * (2 + 2 * r) + 4 * case["rows"]
        if case["direction"] == "train":        # dy, ds, s; dx
            count += n * e * (3 + r)
        return {"bytes": count, "flops": (14 if case["direction"] == "train" else 5) * n}
    shapes = _shapes(case)
    return {"bytes": 2 * e * sum(r * c for r, c in shapes), "flops": _products(shapes)}


# ------------------------------------------------------------------ 64 bits
def _exact_embedding(s):
    T, V, D = s["tokens"], s["vocab"], s["width"]
    f, ids, keep = torch.float64, s["ids"].tolist(), []
    out = torch.zeros(T, D, dtype=f, device="cuda")
    keep = torch.tensor([i for i, v in enumerate(ids) if 0 <= v < V], dtype=torch.long, device="cuda")
    out[keep] = s["weights"].to(f)[s["ids"].long()[keep]] * s["scale"]
    if s["direction"] == "forward":
        return {"out": out}
    # each row's sum as a difference of running sums over the tokens in the order of their ids
    which, order = torch.sort(s["ids"].long()[keep], stable=True)
    grad = torch.zeros(V, D, dtype=f, device="cuda")
    if len(which):
        names, sizes = torch.unique_consecutive(which, return_counts=True)
        ends = torch.cumsum(sizes, 0) - 1
        for c in range(0, D, 256):
            sums = torch.cumsum(s["dout"][:, c:c + 256].to(f)[keep[order]], 0)[ends]
            grad[names, c:c + 256] = torch.diff(sums, dim=0, prepend=torch.zeros_like(sums[:1])) * s["scale"]
    return {"out": out, "dtable": grad}


def _exact_norm(s):
    f, rows, cols = torch.float64, s["rows"], s["cols"]
    train, upload = s["direction"] == "train", s["direction"] == "upload"
    w = s["w"].to(f)
    parts, dw = [], torch.zeros(cols, dtype=f, device="cuda")
    step = max(1, (1 << 26) // cols)
    for i in range(0, rows, step):
        x = s["x"][i:i + step]
        total = x.to(f)
        if s["residual"] is not None:
            total = (total + s["residual"][i:i + step].to(f)).to(x.dtype).to(f)
        r = (torch.linalg.vector_norm(total, dim=1) ** 2 / cols + EPS) ** -0.5
        y = torch.einsum("ij,i,j->ij", total, r, w)
        part = {"s": total, "y": y, "r": r}
        if upload:
            blocks = [y[:, c:c + 32] for c in range(0, cols, 32)]
            q = []
            for b in blocks:
                e = torch.log2(b.abs().amax(1, keepdim=True).clamp(min=2.0 ** -140) / 448).ceil().clamp(-127, 127)
                q.append((b / 2 ** e).float().to(torch.float8_e4m3fn).to(f) * 2 ** e)
            part = {"s": total, "y": torch.cat(q, 1)}
        if train:
            dy = s["dy"][i:i + step].to(f)
            dot = torch.einsum("ij,ij,j->i", dy, total, w) / cols
            part["dx"] = torch.einsum("ij,i,j->ij", dy, r, w) - torch.einsum("ij,i->ij", total, r ** 3 * dot)
            if s["ds"] is not None:
                part["dx"] += s["ds"][i:i + step].to(f)
            dw += torch.einsum("ij,ij,i->j", dy, total, r)
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if train:
        out["dw"] = dw
    return out


def _exact_orthogonalize(u):
    """The same polynomial on the other side of X, X (a + b A + c A A) with A = X^T X of the narrow side."""
    a, b, c = COEFFICIENTS
    tall = u.shape[0] >= u.shape[1]
    x = (u if tall else u.t()).double()
    x = x / (torch.linalg.matrix_norm(x) + NORM_EPS)
    one = torch.eye(x.shape[1], dtype=x.dtype, device=x.device)
    for _ in range(STEPS):
        A = x.t() @ x
        x = x @ (a * one + A @ (b * one + c * A))
    return x if tall else x.t()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalize":
        return [_exact_orthogonalize(u) for u in s["updates"]]
    return _exact_embedding(s) if case["op"] == "embedding" else _exact_norm(s)
