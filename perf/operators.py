"""Cases that time the operators of transformer blocks trained on long or packed
sequences: attention with modified scores (tanh cap, distance bias, document and
prefix masks), the learned relative position bias by buckets with its gradient,
and counter-based dropout around a residual.

``run`` computes a case in plain torch operations (``own`` false) or through the
package's entry points (``own`` true).  ``exact`` gives the same outputs from the
definitions in 64 bits.

Definitions.  For query i and key j of one sequence and head,
    s_ij = scale * q_i . k_j;    with a cap c:  s_ij <- c tanh(s_ij / c)
    s_ij <- s_ij + bias(j - i)   bias(d) = -slope_h |d|, or table[h][buckets[clamp(d, -R, R) + R]]
    pair (i, j) is allowed when (not causal, or j <= i, or j < prefix_b) and, with
    documents, when both tokens have the same id >= 0 (a negative id is padding);
    P = softmax over the allowed j (all zero in a row that allows none), O = P V.
Dropout: elements 8 g .. 8 g + 7 (row-major) take the eight 16-bit halves, low half
first, of the four words of Philox4x32-10 with counter (g, call) and key seed; an
element is kept when its half is >= round(65536 p) and then scaled by
65536 / (65536 - round(65536 p)).
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


def _attention(name, direction, dtype, B, L, H, KV, D, causal=False, cap=0.0, bias="none", buckets=0, reach=0, documents=0,
               padded=False, prefix=False, packed=True):
    """One attention case.  documents: mean length of packed documents (0: none); padded: sequences of L/4 to L
    tokens padded to L; prefix: each sequence has a prefix that every query sees; packed: q, k, v are views of
    one projection."""
    return {"name": name, "op": "attention", "direction": direction, "dtype": dtype, "B": B, "L": L, "H": H, "KV": KV, "D": D,
            "causal": causal, "cap": cap, "bias": bias, "buckets": buckets, "reach": reach, "documents": documents,
            "padded": padded, "prefix": prefix, "packed": packed}


def _dropout(name, direction, dtype, rows, cols, p):
    return {"name": name, "op": "dropout", "direction": direction, "dtype": dtype, "rows": rows, "cols": cols, "p": p}


def listed():
    return [
        # a batch of sequences of one token each: nothing but latency
        _attention("attention one token", "forward", "bf16", 32, 1, 8, 8, 64, bias="bucket", buckets=32, reach=128),
        # the transformer workload's batch (32 sequences of 32..128 tokens padded to 128, 8 heads of 64): one training
        # step of an encoder layer with a learned relative bias
        _attention("attention padded 128", "train", "bf16", 32, 128, 8, 8, 64, bias="bucket", buckets=32, reach=128, padded=True),
        # an encoder layer on whole sequences of 512
        _attention("attention encoder 512", "train", "bf16", 16, 512, 8, 8, 64, bias="bucket", buckets=32, reach=128),
        # a decoder layer with capped scores and shared key heads
        _attention("attention capped 2048", "train", "bf16", 4, 2048, 16, 4, 128, causal=True, cap=50.0, packed=False),
        # short documents packed into one long sequence, distance bias
        _attention("attention documents 8192", "train", "bf16", 1, 8192, 8, 8, 64, causal=True, bias="distance", documents=1000),
        # scoring with a visible prefix at an odd length
        _attention("attention prefix 4095", "forward", "bf16", 2, 4095, 16, 2, 128, causal=True, cap=30.0, prefix=True),
        # the longest sequence, learned bias, shared key heads
        _attention("attention long 16384", "train", "bf16", 1, 16384, 8, 2, 128, causal=True, bias="bucket", buckets=32, reach=128),
        # single precision, as a parity run trains it: small and ragged, then larger
        _attention("attention f32 200", "train", "f32", 4, 200, 4, 4, 32, bias="bucket", buckets=16, reach=64, padded=True),
        _attention("attention f32 1000", "train", "f32", 2, 1000, 8, 8, 64, causal=True, bias="distance", packed=False),
        # the residual branch of the transformer workload's batch: 32 x 128 tokens, width 512
        _dropout("dropout 4096x512", "forward", "bf16", 4096, 512, 0.1),
        # the gradient through it for a large batch
        _dropout("dropout gradient 65536x2048", "gradient", "bf16", 65536, 2048, 0.1),
        # single precision, odd width
        _dropout("dropout f32 1000x777", "forward", "f32", 1000, 777, 0.25),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.3:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows, cols = _log_int(rng, 1, 32768), _log_int(rng, 8, 4096)
        if rng.random() < 0.5:
            cols = max(8, cols // 8 * 8)
        c = _dropout("", rng.choice(["forward", "gradient"]), dtype, rows, cols, rng.choice([0.05, 0.1, 0.25, 0.5]))
    else:
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        direction = rng.choice(["forward", "train", "train"])
        KV = rng.choice([1, 2, 4, 8])
        H = KV * rng.choice([1, 1, 2, 4])
        D = rng.choice([32, 40, 64, 64, 64, 80, 96, 128, 128] if dtype == "bf16" else [16, 32, 48, 64, 128])
        room = 8 * 16384 * 16384 // 2 if dtype == "bf16" else 24 * 1000 * 1000
        # a training step has two tokens at least: the scores' gradient of a lone key is zero
        L = _log_int(rng, 1 if direction == "forward" else 2, min(12000 if dtype == "bf16" else 1200, math.isqrt(room // H)))
        B = _log_int(rng, 1, max(1, min(32, room // (L * L * H))))
        bias = rng.choice(["none", "distance", "bucket", "bucket"])
        buckets = rng.choice([8, 16, 32, 64]) if bias == "bucket" else 0
        reach = _log_int(rng, buckets, 512) if bias == "bucket" else 0
        causal = rng.random() < 0.6
        kind = rng.choice(["none", "none", "documents", "padded"])
        c = _attention("", direction, dtype, B, L, H, KV, D, causal=causal, cap=rng.choice([0.0, 0.0, 20.0, 50.0]), bias=bias,
                       buckets=buckets, reach=reach, documents=_log_int(rng, 16, 2000) if kind == "documents" else 0,
                       padded=kind == "padded", prefix=causal and rng.random() < 0.3, packed=rng.random() < 0.5)
    del c["name"]
    return c


def _bucket_map(buckets, reach, causal):
    """Bucket of each clamped distance d = j - i in -reach..reach: small distances have a bucket each, larger ones
    share logarithmic ranges; without a causal mask the two signs have half of the buckets each."""
    half = buckets if causal else buckets // 2
    near = max(1, half // 2)
    out = []
    for d in range(-reach, reach + 1):
        n = max(-d, 0) if causal else abs(d)
        if n < near:
            b = n
        else:
            b = near + int(math.log(n / near) / max(math.log(max(reach, near + 1) / near), 1e-9) * (half - near))
        b = min(b, half - 1)
        out.append(b if causal or d <= 0 else b + half)
    return np.array(out, np.uint8)


def _documents(case, seed):
    """Document id of each token, int32 [B, L], or None."""
    B, L = case["B"], case["L"]
    if not case["documents"] and not case["padded"]:
        return None
    rng = random.Random(seed * 7919 + 11)
    ids = np.full((B, L), -1, np.int32)
    for b in range(B):
        if case["padded"]:
            ids[b, : rng.randint(max(min(2, L), L // 4), L)] = 0
            continue
        end, at, n = L - rng.randint(0, L // 20), 0, 0
        while at < end:
            size = max(1, int(rng.uniform(0.2, 1.8) * case["documents"]))
            ids[b, at:min(at + size, end)] = n
            at, n = at + size, n + 1
    return ids


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g, dtype=torch.float32).to(t)

    s = dict(case)
    if case["op"] == "dropout":
        rows, cols = case["rows"], case["cols"]
        s["x"] = randn(rows, cols)
        s["residual"] = randn(rows, cols) if case["direction"] == "forward" else None
        s["seed"], s["call"] = (seed * 0x9E3779B97F4A7C15 + 12345) % 2**63, seed % 1000003
        return s
    B, L, H, KV, D = (case[k] for k in ("B", "L", "H", "KV", "D"))
    if case["packed"]:
        qkv = randn(B, L, H + 2 * KV, D)
        s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + KV], qkv[:, :, H + KV:]
    else:
        s["q"], s["k"], s["v"] = randn(B, L, H, D), randn(B, L, KV, D), randn(B, L, KV, D)
    s["dout"] = randn(B, L, H, D) if case["direction"] == "train" else None
    s["slopes"] = s["table"] = s["buckets"] = s["bucket_index"] = s["documents"] = s["prefix"] = None
    if case["bias"] == "distance":
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda")
    if case["bias"] == "bucket":
        s["table"] = (0.5 * torch.randn(H, case["buckets"], device="cuda", generator=g)).to(t)
        s["buckets"] = _bucket_map(case["buckets"], case["reach"], case["causal"])
        s["bucket_index"] = torch.from_numpy(s["buckets"].astype(np.int64)).cuda()
    ids = _documents(case, seed)
    if ids is not None:
        s["documents"] = torch.from_numpy(ids).cuda()
    if case["prefix"]:
        rng = random.Random(seed * 31 + 5)
        s["prefix"] = torch.tensor([rng.randint(0, L // 2) for _ in range(B)], dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms
def _plain_attention(s):
    B, L, H, KV, D = (s[k] for k in ("B", "L", "H", "KV", "D"))
    G, t, scale, cap = H // KV, TYPES[s["dtype"]], s["D"] ** -0.5, s["cap"]
    q = s["q"].float().permute(0, 2, 1, 3).reshape(B, KV, G, L, D)
    k = s["k"].float().permute(0, 2, 1, 3).unsqueeze(2)
    v = s["v"].float().permute(0, 2, 1, 3).unsqueeze(2)
    x = torch.matmul(q, k.transpose(-1, -2)) * scale
    slope = None
    if cap:
        x = torch.tanh(x / cap)
        slope = 1 - x * x if s["direction"] == "train" else None
        x = x * cap
    at = torch.arange(L, device=x.device)
    distance = at[None, :] - at[:, None]
    if s["slopes"] is not None:
        x = x - s["slopes"].view(KV, G, 1, 1) * distance.abs()
    if s["table"] is not None:
        R = s["reach"]
        x = x + s["table"].float()[:, s["bucket_index"][distance.clamp(-R, R) + R]].view(KV, G, L, L)
    allowed = torch.ones(1, 1, 1, L, L, dtype=torch.bool, device=x.device)
    if s["causal"]:
        allowed = (distance <= 0).view(1, 1, 1, L, L)
        if s["prefix"] is not None:
            allowed = allowed | (at < s["prefix"][:, None]).view(B, 1, 1, 1, L)
    if s["documents"] is not None:
        ids = s["documents"]
        allowed = allowed & ((ids[:, :, None] == ids[:, None, :]) & (ids >= 0)[:, :, None]).view(B, 1, 1, L, L)
    x = x.masked_fill(~allowed, float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    del x
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, v)
    out = {"o": o.reshape(B, H, L, D).permute(0, 2, 1, 3).to(t)}
    if s["direction"] == "forward":
        return out
    do = s["dout"].float().permute(0, 2, 1, 3).reshape(B, KV, G, L, D)
    out["dv"] = torch.matmul(p.transpose(-1, -2), do).sum(2).permute(0, 2, 1, 3).to(t)
    dp = torch.matmul(do, v.transpose(-1, -2))
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    del p, dp
    if s["table"] is not None:
        # rows of length 2 L read as rows of length 2 L + 1: column c holds distance c, or c - (2 L + 1); the columns'
        # sums are then gathered into buckets
        e = ds.new_zeros(H, L * (2 * L + 1))
        e[:, :2 * L * L].view(H, L, 2 * L)[:, :, :L] = ds.sum(0).view(H, L, L)
        e = e.view(H, L, 2 * L + 1).sum(1)
        far = torch.arange(2 * L + 1, device=e.device)
        far = torch.where(far < L, far, far - (2 * L + 1))
        hot = s["bucket_index"][far.clamp(-s["reach"], s["reach"]) + s["reach"]][:, None] == torch.arange(s["table"].shape[1], device=e.device)
        out["dtable"] = torch.matmul(e, hot.float()).to(t)
        del e
    if slope is not None:
        ds = ds * slope
    out["dq"] = (torch.matmul(ds, k) * scale).reshape(B, H, L, D).permute(0, 2, 1, 3).to(t)
    out["dk"] = (torch.matmul(ds.transpose(-1, -2), q).sum(2) * scale).permute(0, 2, 1, 3).to(t)
    return out


def _mul_hi_lo(a, m):
    """High and low words of the product of 32-bit words held in int64 (the product wraps, its bits do not change)."""
    x = a * m
    return (x >> 32) & 0xFFFFFFFF, x & 0xFFFFFFFF


def _philox(g, call, k0, k1, rounds=10):
    c0, c1, c2, c3 = g & 0xFFFFFFFF, g >> 32, torch.full_like(g, call & 0xFFFFFFFF), torch.full_like(g, call >> 32)
    for _ in range(rounds):
        h0, l0 = _mul_hi_lo(c0, 0xD2511F53)
        h1, l1 = _mul_hi_lo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], 1)


def _plain_dropout(s):
    x = s["x"]
    n, drop = x.numel(), round(65536 * s["p"])
    g = torch.arange((n + 7) // 8, device=x.device)
    bits = _philox(g, s["call"], s["seed"] & 0xFFFFFFFF, s["seed"] >> 32).reshape(-1)[:n].view(x.shape)
    y = torch.where(bits >= drop, x.float() * (65536 / (65536 - drop)), torch.zeros((), device=x.device))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


def run(s):
    if not own:
        return {"y": _plain_dropout(s)} if s["op"] == "dropout" else _plain_attention(s)
    from paper_2504_13850_gb300 import api

    if s["op"] == "dropout":
        if s["direction"] == "gradient":
            return {"y": api.dropout_grad(s["x"], s["p"], s["seed"], s["call"])}
        return {"y": api.dropout_add(s["x"], s["residual"], s["p"], s["seed"], s["call"])}
    how = {"causal": s["causal"], "softcap": s["cap"], "slopes": s["slopes"], "table": s["table"], "buckets": s["buckets"],
           "documents": s["documents"], "prefix": s["prefix"]}
    o, lse = api.attention_forward(s["q"], s["k"], s["v"], **how)
    if s["direction"] == "forward":
        return {"o": o}
    dq, dk, dv, dtable = api.attention_backward(s["dout"], s["q"], s["k"], s["v"], o, lse, **how)
    out = {"o": o, "dq": dq, "dk": dk, "dv": dv}
    if dtable is not None:
        out["dtable"] = dtable
    return out


def _pairs(case):
    """Allowed (query, key) pairs of the whole batch (documents as one seed lays them out; prefixes at their mean)."""
    B, L = case["B"], case["L"]
    ids = _documents(case, 0)
    runs = [(b, n) for b in range(B) for n in ([L] if ids is None else np.unique(ids[b][ids[b] >= 0], return_counts=True)[1].tolist())]
    pairs = sum(n * (n + 1) / 2 if case["causal"] else n * n for _, n in runs)
    if case["prefix"]:
        pairs += B * (L / 4) ** 2 / 2
    return pairs


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * (3 if case["direction"] == "forward" else 2), "flops": 2 * n}
    B, L, H, KV, D = (case[k] for k in ("B", "L", "H", "KV", "D"))
    train = case["direction"] == "train"
    wide, narrow = B * L * H * D * e, B * L * KV * D * e
    # forward reads q, k, v and writes o; a training step also reads dout and writes dq, dk, dv
    return {"bytes": (2 * wide + 2 * narrow) + (2 * wide + 2 * narrow if train else 0),
            "flops": (14 if train else 4) * _pairs(case) * H * D}


# ------------------------------------------------------------------ 64 bits
def _exact_attention(case, seed):
    s = prepare(case, seed)
    B, L, H, KV, D = (case[k] for k in ("B", "L", "H", "KV", "D"))
    dev, f = s["q"].device, torch.float64
    train = case["direction"] == "train"
    out = {"o": torch.zeros(B, L, H, D, dtype=f, device=dev)}
    if train:
        out["dq"] = torch.zeros(B, L, H, D, dtype=f, device=dev)
        out["dk"], out["dv"] = (torch.zeros(B, L, KV, D, dtype=f, device=dev) for _ in range(2))
        if case["bias"] == "bucket":
            out["dtable"] = torch.zeros(H, case["buckets"], dtype=f, device=dev)
    pos = torch.arange(L, device=dev)
    step = max(1, (1 << 27) // L)                                   # query rows at a time
    for b in range(B):
        for h in range(H):
            c = h // (H // KV)
            K, V = s["k"][b, :, c].to(f), s["v"][b, :, c].to(f)
            for r in range(0, L, step):
                Q, rows = s["q"][b, r:r + step, h].to(f), pos[r:r + step, None]
                z = Q @ K.T / math.sqrt(D)
                w = torch.tanh(z / case["cap"]) if case["cap"] else None
                z = z if w is None else case["cap"] * w
                d = pos[None, :] - rows
                if case["bias"] == "distance":
                    z = z - float(s["slopes"][h]) * d.abs()
                if case["bias"] == "bucket":
                    which = s["bucket_index"][torch.clamp(d, -case["reach"], case["reach"]) + case["reach"]]
                    z = z + s["table"][h].to(f)[which]
                ok = d <= (0 if case["causal"] else L)
                if case["prefix"]:
                    ok = ok | (pos < int(s["prefix"][b]))[None, :]
                if s["documents"] is not None:
                    mine = s["documents"][b, r:r + step, None]
                    ok = ok & (mine >= 0) & (mine == s["documents"][b][None, :])
                z = torch.where(ok, z, torch.full_like(z, -math.inf))
                P = torch.nan_to_num(torch.softmax(z, 1))           # a row that allows no key: zeros
                out["o"][b, r:r + step, h] = P @ V
                if not train:
                    continue
                dO = s["dout"][b, r:r + step, h].to(f)
                out["dv"][b, :, c] += P.T @ dO
                J = dO @ V.T
                S = P * J - P * (P * J).sum(1, keepdim=True)
                if case["bias"] == "bucket":
                    for n in range(case["buckets"]):
                        out["dtable"][h, n] += (S * (which == n)).sum()
                if w is not None:
                    S = S * (1 - w ** 2)
                out["dq"][b, r:r + step, h] = S @ K / math.sqrt(D)
                out["dk"][b, :, c] += S.T @ Q / math.sqrt(D)
    return out


def _exact_dropout(case, seed):
    s = prepare(case, seed)
    x = s["x"].double().cpu().numpy().reshape(-1)
    M = np.uint64(0xFFFFFFFF)
    g = np.arange((x.size + 7) // 8, dtype=np.uint64)
    w = [g & M, g >> np.uint64(32), np.full_like(g, s["call"] & 0xFFFFFFFF), np.full_like(g, s["call"] >> 32)]
    key = [s["seed"] & 0xFFFFFFFF, s["seed"] >> 32]
    for _ in range(10):
        a, b = w[0] * np.uint64(0xD2511F53), w[2] * np.uint64(0xCD9E8D57)
        w = [(b >> np.uint64(32)) ^ w[1] ^ np.uint64(key[0]), b & M, (a >> np.uint64(32)) ^ w[3] ^ np.uint64(key[1]), a & M]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = np.stack([v for x4 in w for v in (x4 & np.uint64(0xFFFF), x4 >> np.uint64(16))], 1).reshape(-1)[: x.size]
    drop = round(65536 * case["p"])
    y = np.where(halves >= drop, x * 65536.0 / (65536 - drop), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].double().cpu().numpy().reshape(-1)
    return {"y": torch.from_numpy(y.reshape(case["rows"], case["cols"]))}


def exact(case, seed):
    if case["op"] == "dropout":
        return _exact_dropout(case, seed) if case["rows"] * case["cols"] <= 1 << 27 else None
    if case["B"] * case["H"] * case["L"] ** 2 * case["D"] > 1 << 39:
        return None
    return _exact_attention(case, seed)
