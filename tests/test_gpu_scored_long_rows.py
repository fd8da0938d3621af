"""Rows of very many keys on the bf16 path, with values and gradients of mean 1, so
that O and D are large beside what the gradients of queries are made of: sampled
rows against 64 bits.  The bounds: each product's operands (P, dS) carry roundings
to bf16 that are independent of each other, the accumulator of the tensor cores
truncates once per 16 keys (2^-23 of the sum), D is granted no error but that of
fp32 sums; D from the stored O fails."""
import numpy as np
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
U, F, ACC = R.ROUND[BF], R.FP32, 2.0 ** -20


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


@pytest.mark.parametrize("L,D", [(1000, 64), (16384, 64), (16384, 128), (100001, 64), (60000, 128)])
def test_sampled_rows(L, D):
    g = torch.Generator(device="cuda").manual_seed(L)

    def rnd(mean):
        return (mean + torch.randn(1, L, 1, D, device="cuda", generator=g)).to(BF)

    x = [rnd(0), rnd(0), rnd(1)]
    dout = rnd(1)
    table, buckets = (0.5 * torch.randn(1, 8, device="cuda", generator=g)).to(BF), api.relative_buckets(8, 100)
    o, lse = api.attention_forward(*x, table=table, buckets=buckets)
    dq, dk, dv, dtable = api.attention_backward(dout, *x, o, lse, table=table, buckets=buckets)
    api.attention_error()
    at = torch.randint(0, L, (24,), device="cuda", generator=g)
    Q, K, V, dO, O = (t[0, :, 0].double() for t in (*x, dout, o))
    which = torch.from_numpy(buckets.astype(np.int64)).cuda()
    d = (torch.arange(L, device="cuda")[None] - at[:, None]).clamp(-100, 100)
    s, truncation = D ** -0.5, 2.0 ** -23 * (L / 16 + 16)
    z = s * Q[at] @ K.T + table[0].double()[which[d + 100]]
    P = torch.softmax(z, -1)
    assert bool(((lse[0, 0, at].double() - torch.logsumexp(z, -1)).abs() <= F * (1 + lse[0, 0, at].abs())).all())
    want, sums = P @ V, P @ V.abs()
    assert bool(((O[at] - want).abs() <= (U + F + truncation) * sums + U * want.abs()).all())
    dP, dP_abs = dO[at] @ V.T, dO[at].abs() @ V.abs().T
    exact, stored = (P * dP).sum(-1, keepdim=True), (dO[at] * O[at]).sum(-1, keepdim=True)
    dS, off = P * (dP - exact), (exact - stored).abs()
    want = s * dS @ K
    # dS as it enters the product is P (dP - D0), and P times what D0 is off by is taken off after it
    roundings = U * (((dS.abs() + P * off) ** 2 @ K ** 2).sqrt().norm(dim=1) + ((off * P) ** 2 @ K ** 2).sqrt().norm(dim=1))
    sums = ((F * dS.abs() + ACC * P * (dP_abs + exact.abs())) @ K.abs()).norm(dim=1)
    partial = ((dS.abs() + 2 * off * P) ** 2 @ K ** 2).sqrt().norm(dim=1) + 2 * off[:, 0] * (P @ K).norm(dim=1)
    bound = s * (roundings + sums + truncation * partial) + U * want.norm(dim=1)
    assert bool(((dq[0, at, 0].double() - want).norm(dim=1) <= bound).all())
    planted = s * (P * (dP - stored)) @ K
    assert L < 10000 or bool(((planted - want).norm(dim=1) > bound).any())
    # the same rows as keys: P^T from every query, whose lse has been looked at above
    zt = s * K[at] @ Q.T + table[0].double()[which[100 - d]]
    Pt = torch.exp(zt - lse[0, 0].double()[None])
    want, sums = Pt @ dO, Pt @ dO.abs()
    assert bool(((dv[0, at, 0].double() - want).abs() <= (U + F + truncation) * sums + U * want.abs()).all())
