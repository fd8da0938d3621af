"""Plain 64-bit implementations that the operator tests compare against:
attention with modified scores (with error bounds derived from the stored
precision) and Philox dropout."""
import numpy as np
import torch

# Unit roundoff (2 ** -p for p significant bits) of the type that P, dS and the outputs are rounded to.
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
# Relative error that fp32 arithmetic may leave in a score's exponential and in
# the sums: scores of magnitude up to ~50 carry ~4 roundings of 2^-24 each
# (~1.2e-5 in the exponent), sums of a few thousand terms ~1e-5.
FP32 = 4e-5


def attention(q, k, v, dout=None, causal=False, softcap=0.0, scale=None, slopes=None, table=None, buckets=None,
              documents=None, prefix=None):
    """(values, bounds): dicts with o, lse and, with dout, dq, dk, dv, dtable
    in 64 bits, and elementwise error bounds of an implementation that holds
    sums in fp32 and rounds P, dS and the outputs once to q's type.

    Each bound follows the product that forms the output, with u the roundoff
    and f = FP32: |do| <= (u + f) P |v| + u |o|;  D = dO . o inherits that
    error; |d(dS)| <= u |dS| + f P (|dP| + |D|) + P |dD|; and so on."""
    u, f = ROUND[q.dtype], FP32
    B, L, H, D = q.shape
    KV, dev = k.shape[2], q.device
    G = H // KV
    scale = D ** -0.5 if scale is None else scale
    pos = torch.arange(L, device=dev)
    dist = pos[None, :] - pos[:, None]
    ok = (dist <= 0 if causal else torch.ones_like(dist, dtype=torch.bool))[None].expand(B, L, L)
    if prefix is not None:
        ok = ok | (pos[None, None, :] < prefix.long()[:, None, None])
    live = torch.ones(B, L, dtype=torch.bool, device=dev)
    if documents is not None:
        live = documents >= 0
        ok = ok & (documents[:, :, None] == documents[:, None, :]) & live[:, :, None]

    def heads(t, n):          # [B, heads, L, D]; what padding holds must not matter
        t = t.double().permute(0, 2, 1, 3)
        t = torch.where(live[:, None, :, None], t, torch.zeros_like(t))
        return t.repeat_interleave(n, 1)

    Q, K, V = heads(q, 1), heads(k, G), heads(v, G)
    z = scale * Q @ K.mT
    chain = torch.ones_like(z)
    if softcap:
        t = torch.tanh(z / softcap)
        z, chain = softcap * t, 1 - t * t
    if slopes is not None:
        z = z - slopes.double()[None, :, None, None] * dist.abs()
    if table is not None:
        R = buckets.size // 2
        which = torch.from_numpy(buckets.astype(np.int64)).to(dev)[dist.clamp(-R, R) + R]
        z = z + table.double()[:, which][None]
    z = z.masked_fill(~ok[:, None], float("-inf"))
    lse = torch.logsumexp(z, -1)
    P = torch.where(ok[:, None], torch.exp(z - lse.masked_fill(torch.isinf(lse), 0.0)[..., None]), torch.zeros_like(z))
    O = P @ V
    e_o = (u + f) * (P @ V.abs()) + u * O.abs()

    def back(t):
        return t.permute(0, 2, 1, 3)

    def grouped(t):
        return t.reshape(B, KV, G, L, D).sum(2).permute(0, 2, 1, 3)

    val = {"o": back(O), "lse": lse}
    err = {"o": back(e_o), "lse": f * (1 + lse.abs())}
    if dout is None:
        return val, err
    dO = heads(dout, 1)
    dP, dP_abs = dO @ V.mT, dO.abs() @ V.abs().mT
    Dl = (dO * O).sum(-1, keepdim=True)
    e_D = (dO.abs() * (e_o + f * O.abs())).sum(-1, keepdim=True)
    dS = P * (dP - Dl)
    e_S = u * dS.abs() + P * (f * (dP_abs + Dl.abs()) + e_D)          # of dS as it enters a product
    e_T = P * (f * (dP_abs + Dl.abs()) + e_D)                           # of dS as it is summed in fp32
    if table is not None:
        nb = table.shape[1]
        hot = torch.nn.functional.one_hot(which, nb).double()
        val["dtable"] = torch.einsum("bhij,ijn->hn", dS, hot)
        err["dtable"] = torch.einsum("bhij,ijn->hn", e_T + f * dS.abs(), hot) + u * val["dtable"].abs()
    dS, e_S = dS * chain, e_S * chain.clamp_min(f)
    val["dv"], val["dq"], val["dk"] = grouped(P.mT @ dO), back(scale * dS @ K), grouped(scale * dS.mT @ Q)
    err["dv"] = grouped((u + f) * P.mT @ dO.abs()) + u * val["dv"].abs()
    err["dq"] = back(scale * (e_S + f * dS.abs()) @ K.abs()) + u * val["dq"].abs()
    err["dk"] = grouped(scale * (e_S + f * dS.abs()).mT @ Q.abs()) + u * val["dk"].abs()
    return val, err


def philox(counter, key):
    """Philox4x32-10: four words for each row of counter (uint64 [n, 4] of 32-bit values)."""
    M = np.uint64(0xFFFFFFFF)
    s32 = np.uint64(32)
    c = [counter[:, i].astype(np.uint64) for i in range(4)]
    k = list(key)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ np.uint64(k[0]), b & M, (a >> s32) ^ c[3] ^ np.uint64(k[1]), a & M]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1)


def dropout_mask(n, p, seed, call):
    """(keep [n], scale) of the framework's dropout."""
    g = np.arange((n + 7) // 8, dtype=np.uint64)
    M, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    ctr = np.stack([g & M, g >> s32, np.full_like(g, call & 0xFFFFFFFF), np.full_like(g, call >> 32)], 1)
    w = philox(ctr, (seed & 0xFFFFFFFF, seed >> 32))
    half = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(-1)[:n]
    drop = round(65536 * p)
    return half >= drop, (65536.0 / (65536 - drop) if drop < 65536 else 0.0)
