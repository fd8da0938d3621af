"""The D of the bf16 backward pass.  D = dO . O taken from the stored O carries O's
rounding, which leaves every row of dS with a sum that is not zero; dK and the
table gradient come from a corrected D, dQ as well where a tile of 128 queries
walks at most two blocks of 64 keys.  The values here make that rounding large
(V has a mean of 16, so O's mean over keys vanishes in it), and the bounds grant
no error of D; the same formulas with D from the stored O fail them."""
import numpy as np
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
U, F = R.ROUND[BF], R.FP32
# fp32 accumulation of dP and of the row sums: a few units of 2^-23 of the sums of absolute values
ACC = 2.0 ** -20


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


def inputs(L, D, seed, documents=None):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(mean, size):
        return (mean + size * torch.randn(1, L, 2, D, device="cuda", generator=g)).to(BF)

    x = {"q": rnd(0, 1), "k": rnd(0, 1), "v": rnd(16, 1), "dout": rnd(1, 1)}
    how = {"table": torch.randn(2, 8, device="cuda", generator=g).to(BF), "buckets": api.relative_buckets(8, 8)}
    if documents is not None:
        how["documents"] = torch.tensor(documents, dtype=torch.int32, device="cuda").view(1, L)
    return x, how


def run(x, how):
    o, lse = api.attention_forward(x["q"], x["k"], x["v"], **how)
    dq, dk, dv, dtable = api.attention_backward(x["dout"], x["q"], x["k"], x["v"], o, lse, **how)
    api.attention_error()
    return {"o": o, "dq": dq, "dk": dk, "dtable": dtable}


def parts(x, how, o):
    """64-bit Q, K [H, L, D], P, dP's absolute sums, D, D from the stored o, dS, and dS with that D; the pairs' buckets."""
    Q, K, V, dO, O = (t[0].double().transpose(0, 1) for t in (x["q"], x["k"], x["v"], x["dout"], o))
    L, D = Q.shape[1:]
    pos = torch.arange(L, device="cuda")
    reach = how["buckets"].size // 2
    which = torch.from_numpy(how["buckets"].astype(np.int64)).cuda()[(pos[None] - pos[:, None]).clamp(-reach, reach) + reach]
    z = D ** -0.5 * Q @ K.mT + how["table"].double()[:, which]
    if "documents" in how:
        z = z.masked_fill(how["documents"][0][:, None] != how["documents"][0][None], float("-inf"))
    P = torch.softmax(z, -1)
    dP = dO @ V.mT
    exact, stored = (P * dP).sum(-1, keepdim=True), (dO * O).sum(-1, keepdim=True)
    return Q, K, P, dO.abs() @ V.abs().mT, exact, P * (dP - exact), P * (dP - stored), which


def gradients(dS, Q, K, which):
    hot = torch.nn.functional.one_hot(which, 8).double()
    s = Q.shape[2] ** -0.5
    return {"dq": s * dS @ K, "dk": s * dS.mT @ Q, "dtable": torch.einsum("hij,ijn->hn", dS, hot)}


def bounds(P, dP_abs, D, dS, Q, K, which):
    """dq, dk: 2-norms per head.  dS's roundings to bf16 are independent, so their
    errors add as squares; the relative error of P and the accumulations are taken
    in full.  dtable: elementwise, dS is summed in fp32."""
    s, acc = Q.shape[2] ** -0.5, ACC * P * (dP_abs + D.abs())
    hot = torch.nn.functional.one_hot(which, 8).double()
    g = gradients(dS, Q, K, which)

    def norm(t):
        return t.flatten(1).norm(dim=1)

    out = {}
    for name, a, e, X in (("dq", dS.abs(), acc, K.abs()), ("dk", dS.abs().mT, acc.mT, Q.abs())):
        out[name] = s * (U * norm(((a ** 2) @ (X ** 2)).sqrt()) + norm((F * a + e) @ X)) + U * norm(g[name])
    out["dtable"] = torch.einsum("hij,ijn->hn", F * dS.abs() + acc, hot) + U * g["dtable"].abs()
    return out


def error(name, got, want):
    d = (got.double() if name == "dtable" else got[0].double().transpose(0, 1)) - want
    return d.abs() if name == "dtable" else d.flatten(1).norm(dim=1)


@pytest.mark.parametrize("D", [64, 128])
def test_keys_and_table(D):
    x, how = inputs(512, D, seed=D)
    got = run(x, how)
    Q, K, P, dP_abs, exact, dS, dS0, which = parts(x, how, got["o"])
    want, wrong, bound = gradients(dS, Q, K, which), gradients(dS0, Q, K, which), bounds(P, dP_abs, exact, dS, Q, K, which)
    for name in ("dk", "dtable"):
        assert bool((error(name, got[name], want[name]) <= bound[name]).all()), name
        planted = (wrong[name] - want[name]).abs() if name == "dtable" else (wrong[name] - want[name]).flatten(1).norm(dim=1)
        assert bool((planted > bound[name]).any()), name           # the bound tells the two apart


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [40, 64, 65, 128])
def test_queries_of_short_sequences(L, D):
    x, how = inputs(L, D, seed=L + D)
    got = run(x, how)
    Q, K, P, dP_abs, exact, dS, dS0, which = parts(x, how, got["o"])
    want, bound = gradients(dS, Q, K, which), bounds(P, dP_abs, exact, dS, Q, K, which)
    for name in ("dq", "dk", "dtable"):
        assert bool((error(name, got[name], want[name]) <= bound[name]).all()), name
    planted = (gradients(dS0, Q, K, which)["dq"] - want["dq"]).flatten(1).norm(dim=1)
    assert bool((planted > bound["dq"]).any())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("first", [128, 129])
def test_queries_on_either_side_of_two_blocks(first, D):
    """A document of 128 tokens gives the first tile two blocks of keys, one of 129
    three: dQ has the exact D on one side of that edge and O's rounding, within the
    usual bound, on the other."""
    L = 400
    x, how = inputs(L, D, seed=first, documents=[0] * first + [1] * (L - first))
    got = run(x, how)
    ref, err = R.attention(x["q"], x["k"], x["v"], x["dout"], **how)
    assert bool(((got["dq"].double() - ref["dq"]).abs() <= err["dq"]).all())
    y = {n: t[:, :first] for n, t in x.items()}
    Q, K, P, dP_abs, exact, dS, dS0, which = parts(y, {n: t for n, t in how.items() if n != "documents"}, got["o"][:, :first])
    want, bound = gradients(dS, Q, K, which)["dq"], bounds(P, dP_abs, exact, dS, Q, K, which)["dq"]
    if first == 128:
        assert bool((error("dq", got["dq"][:, :first], want) <= bound).all())


def test_backward_on_another_stream():
    """The given stream also carries the copy of a gradient whose innermost stride is not 1."""
    x, how = inputs(200, 64, seed=5)
    x["dout"] = x["dout"].transpose(2, 3).contiguous().transpose(2, 3)
    ref, err = R.attention(x["q"], x["k"], x["v"], x["dout"], **how)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o, lse = api.attention_forward(x["q"], x["k"], x["v"], stream=s.cuda_stream, **how)
    grads = api.attention_backward(x["dout"], x["q"], x["k"], x["v"], o, lse, stream=s.cuda_stream, **how)
    api.attention_error(stream=s.cuda_stream)
    for name, g in zip(("dq", "dk", "dv", "dtable"), grads):
        assert bool(((g.double() - ref[name]).abs() <= err[name]).all()), name


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [100, 512])
@pytest.mark.parametrize("cap", [1.0, 100.0])
def test_queries_under_a_cap(cap, L, D):
    """Under a cap each pair of dS carries the cap's derivative, and so does what D
    was off by: scores of a few units under a cap of 1, and under one of 100."""
    x, how = inputs(L, D, seed=L)
    x["q"] = 2 * x["q"]
    how["softcap"] = cap
    got = run(x, how)
    Q, K, V, dO, O = (t[0].double().transpose(0, 1) for t in (x["q"], x["k"], x["v"], x["dout"], got["o"]))
    pos, reach, s = torch.arange(L, device="cuda"), how["buckets"].size // 2, D ** -0.5
    which = torch.from_numpy(how["buckets"].astype(np.int64)).cuda()[(pos[None] - pos[:, None]).clamp(-reach, reach) + reach]
    t = torch.tanh(s * Q @ K.mT / cap)
    P, chain = torch.softmax(cap * t + how["table"].double()[:, which], -1), 1 - t * t
    dP, dP_abs = dO @ V.mT, dO.abs() @ V.abs().mT
    exact, stored = (P * dP).sum(-1, keepdim=True), (dO * O).sum(-1, keepdim=True)
    dS, off = P * (dP - exact), (exact - stored).abs()
    want = s * (dS * chain) @ K

    def norm(a):
        return a.flatten(1).norm(dim=1)

    # the derivative is held as fp16 (2^-11 of it), then the products' operands as bf16
    operands = [(dS.abs() + P * off) * chain, off * P * chain]
    bound = s * (sum((U + 2.0 ** -11) * norm((a ** 2 @ K ** 2).sqrt()) for a in operands)
                 + norm((chain * (F * dS.abs() + ACC * P * (dP_abs + exact.abs()))) @ K.abs())) + U * norm(want)
    assert bool((error("dq", got["dq"], want) <= bound).all())
    for wrong in (s * (P * (dP - stored) * chain) @ K, want + s * ((exact - stored) * P * (1 - chain)) @ K):
        assert cap > 1 or bool((norm(wrong - want) > bound).any())          # D from the stored O; a correction without the derivative


@pytest.mark.parametrize("D", [20, 36, 100])
@pytest.mark.parametrize("L,cap", [(60, 0.0), (300, 0.0), (300, 1.0), (700, 0.0)])
def test_queries_on_the_cuda_cores(L, cap, D):
    """bf16 widths that the tensor cores do not take: P and dS are not rounded there,
    so only fp32 sums and the last rounding are granted.  Few tiles, which several
    blocks share, and a single one."""
    x, how = inputs(L, D, seed=L + D)
    x["q"] = 2 * x["q"]
    how["softcap"] = cap
    got = run(x, how)
    Q, K, V, dO, O = (t[0].double().transpose(0, 1) for t in (x["q"], x["k"], x["v"], x["dout"], got["o"]))
    pos, reach, s = torch.arange(L, device="cuda"), how["buckets"].size // 2, D ** -0.5
    which = torch.from_numpy(how["buckets"].astype(np.int64)).cuda()[(pos[None] - pos[:, None]).clamp(-reach, reach) + reach]
    z = s * Q @ K.mT
    t = torch.tanh(z / cap) if cap else torch.zeros_like(z)
    P, chain = torch.softmax((cap * t if cap else z) + how["table"].double()[:, which], -1), 1 - t * t
    dP, dP_abs = dO @ V.mT, dO.abs() @ V.abs().mT
    exact, stored = (P * dP).sum(-1, keepdim=True), (dO * O).sum(-1, keepdim=True)
    dS = P * (dP - exact)
    want = s * (dS * chain) @ K

    def norm(a):
        return a.flatten(1).norm(dim=1)

    # 1 - t^2 in fp32 is off by 2^-23 beside its own size
    bound = s * norm((chain * (F * dS.abs() + ACC * P * (dP_abs + exact.abs())) + 2.0 ** -23 * dS.abs()) @ K.abs()) + U * norm(want)
    assert bool((error("dq", got["dq"], want) <= bound).all())
    assert bool((norm(s * (P * (dP - stored) * chain) @ K - want) > bound).any())
