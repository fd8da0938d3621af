"""Attention whose tanh cap is far above the scores, forward and backward,
against the 64-bit implementation: the cap then hardly changes anything, and
neither pass may lose the scores beside it."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build
from test_gpu_scored import check, make

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
CAPS = [64.0, 65.0, 1e3, 1e4, 1e5, 1e6, 1e8]


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 48)])
@pytest.mark.parametrize("L,bias,causal", [(100, "bucket", False), (330, "none", True), (330, "distance", True),
                                           (290, "bucket", True)])
def test_caps_above_the_scores(L, bias, causal, dtype, D, cap):
    check(*make(2, L, 4, 2, D, dtype, seed=3, bias=bias, causal=causal, cap=cap, docs="packed"))


@pytest.mark.parametrize("cap", [100.0, 1e4, 1e6])
@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 64)])
def test_one_row_near_the_cap_among_ordinary_ones(dtype, D, cap):
    """One query's scores come near the cap; those of its neighbours, in the
    same tile, stay ordinary.  Its dout is zero: fp32 holds no probabilities of
    scores that large, the neighbours' bounds are the usual ones."""
    x, how = make(1, 300, 4, 2, D, dtype, seed=7, causal=True, cap=cap)
    i, j, scale = 140, 130, D ** -0.5
    for h in range(4):
        k = x["k"][0, j, h // 2].float()
        x["q"][0, i, h] = (k * (0.8 * cap / (scale * (k * k).sum()))).to(dtype)
    x["dout"][0, i] = 0
    check(x, how)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("D", [64, 96])
def test_scores_beyond_the_cap_in_fp32(D, seed):
    """Scores of several times the cap, where the cap's derivative is small and has to be as exact as the rest."""
    check(*make(6, 112, 4, 2, D, F32, seed=100 + seed, bias="distance", causal=True, cap=2.0, scale=1.0, docs="mixed"))


@pytest.mark.parametrize("y", [3.0, 7.0, 9.0])
@pytest.mark.parametrize("L,D", [(100, 64), (100, 128), (400, 64), (400, 128)])
def test_every_score_beyond_the_cap_in_bf16(L, D, y):
    """All scores are about y times the cap, so that the derivative (down to 6e-8) is all
    that scales dQ and dK.  2-norms per head: P and dS (and what the correction of D
    takes off) are rounded to bf16 and the derivative to fp16, independently of each
    other; the derivative, exp(-2 y) in its exponent, takes the scores' fp32 rounding
    of 8 y 2^-24 at most, and fp32 sums as everywhere."""
    g = torch.Generator(device="cuda").manual_seed(int(10 * y) + L + D)

    def rnd(mean, size):
        return (mean + size * torch.randn(1, L, 2, D, device="cuda", generator=g)).to(BF)

    s = D ** -0.5
    q, k, v, dout = rnd(y / (D * s), 0.0), rnd(1.0, 0.1), rnd(0.0, 1.0), rnd(0.0, 1.0)
    o, lse = api.attention_forward(q, k, v, softcap=1.0)
    dq, dk, _, _ = api.attention_backward(dout, q, k, v, o, lse, softcap=1.0)
    api.attention_error()
    Q, K, V, dO, O = (t[0].double().transpose(0, 1) for t in (q, k, v, dout, o))
    t = torch.tanh(s * Q @ K.mT)
    P, chain = torch.softmax(t, -1), 1 / torch.cosh(s * Q @ K.mT) ** 2
    dP, dP_abs = dO @ V.mT, dO.abs() @ V.abs().mT
    exact = (P * dP).sum(-1, keepdim=True)
    dS, off = P * (dP - exact), (exact - (dO * O).sum(-1, keepdim=True)).abs()
    U, F, u = 2.0 ** -8, 4e-5, 8 * y * 2.0 ** -24

    def norm(a):
        return a.flatten(1).norm(dim=1)

    for got, X, turn in ((dq, K, lambda a: a), (dk, Q, lambda a: a.mT)):
        want = s * turn(dS * chain) @ X
        operands = [(dS.abs() + P * off) * chain] + ([off * P * chain] if turn(dS) is dS else [])
        bound = s * (sum((U + 2.0 ** -11) * norm((turn(a) ** 2 @ X ** 2).sqrt()) for a in operands)
                     + norm(turn(chain * ((F + u) * dS.abs() + 2.0 ** -20 * P * (dP_abs + exact.abs()))) @ X.abs())) + U * norm(want)
        assert bool((norm(got[0].double().transpose(0, 1) - want) <= bound).all())
