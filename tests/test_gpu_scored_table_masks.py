"""A table of which some entries are masks: -1e4, -1e9, the type's lowest value,
minus infinity.  Rows that see nothing else keep a softmax over what they see
(a finite entry counts as -2^15 at least), or nothing at all for infinity."""
import numpy as np
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build
from test_gpu_scored import make

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
END = 32768.0


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


def agree(x, how, loose):
    """Values against the 64-bit implementation with the clamped table.  `loose`
    [B, L]: rows of only masked keys, whose lse of -2^15 + s is held to 2^-24 of
    itself in fp32: P's exponent is off by up to eight such roundings (of the
    score, its scaling, the product and the sum that form lse, lse's scaling, and
    of the constants of both scalings), 8 * 2^-24 * 2^15 = 2^-6, and with it
    everything that row contributes."""
    ref_how = dict(how, table=torch.where(torch.isinf(how["table"]), how["table"], how["table"].float().clamp(-END, END)))
    ref, err = R.attention(x["q"], x["k"], x["v"], x["dout"], **ref_how)
    o, lse = api.attention_forward(x["q"], x["k"], x["v"], **how)
    dq, dk, dv, dtable = api.attention_backward(x["dout"], x["q"], x["k"], x["v"], o, lse, **how)
    api.attention_error()
    # what the loose rows add: the 64-bit gradients of those rows alone, times 2^-6 of
    # the sums of absolute values that form them
    off = 2.0 ** -6
    B, L, H, D = x["q"].shape
    G, scale = H // x["k"].shape[2], D ** -0.5
    rows = loose[:, None, :, None].double()
    V = x["v"].double().permute(0, 2, 1, 3).repeat_interleave(G, 1).abs()
    K = x["k"].double().permute(0, 2, 1, 3).repeat_interleave(G, 1).abs()
    dO = x["dout"].double().permute(0, 2, 1, 3).abs()
    Q = x["q"].double().permute(0, 2, 1, 3).abs()
    # P <= 1 and a loose row sees the same keys as a causal row
    see = torch.tril(torch.ones(L, L, dtype=torch.float64, device="cuda"))
    dS = see * rows * 2 * (dO @ V.mT).amax(-1, keepdim=True)
    more = {"o": off * (rows * (see @ V)).permute(0, 2, 1, 3), "lse": off * loose[:, None].double().expand(B, H, L),
            "dq": off * scale * (dS @ K).permute(0, 2, 1, 3),
            "dk": off * scale * (dS.mT @ Q).reshape(B, -1, G, L, D).sum(2).permute(0, 2, 1, 3),
            "dv": off * ((see * rows).mT @ dO).reshape(B, -1, G, L, D).sum(2).permute(0, 2, 1, 3),
            "dtable": off * dS.sum((0, 2, 3))[:, None].expand(H, how["table"].shape[1])}
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv), ("dtable", dtable)):
        want, bound = ref[name], err[name] + more[name] + 1e-30
        g = got.double()
        ok = ((g - want).abs() <= bound) | (torch.isinf(want) & (g == want))
        assert bool(ok.all()), (name, int((~ok).sum()), float(((g - want).abs() / bound)[~ok].max()))
    return o, lse, dq, dk, dv


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (BF, 20), (F32, 32)])
@pytest.mark.parametrize("mask", [-1e4, -1e9, "lowest"])
@pytest.mark.parametrize("L", [1, 40, 300])
def test_masked_distances(L, mask, dtype, D):
    """Distance 0 is masked (no query sees itself), so the first causal row sees
    only a masked key; then every distance of head 0."""
    x, how = make(2, L, 4, 2, D, dtype, seed=L, bias="bucket", nb=8, reach=20, causal=True)
    value = float(torch.finfo(dtype).min) if mask == "lowest" else mask
    how["table"][:, int(how["buckets"][20])] = value
    loose = torch.zeros(2, L, dtype=torch.bool, device="cuda")
    loose[:, 0] = True
    agree(x, how, loose)
    how["table"][0] = value
    agree(x, how, torch.ones_like(loose))


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 32)])
def test_infinite_entries_mask_entirely(dtype, D):
    x, how = make(2, 300, 4, 2, D, dtype, seed=1, bias="bucket", nb=8, reach=20, causal=True)
    how["table"][:, int(how["buckets"][20])] = float("-inf")
    o, lse, dq, dk, dv = (t.double() for t in agree(x, how, torch.zeros(2, 300, dtype=torch.bool, device="cuda")))
    assert bool((o[:, 0] == 0).all()) and bool((dq[:, 0] == 0).all()) and bool(torch.isinf(lse[:, :, 0]).all())
    assert all(bool(torch.isfinite(t).all()) for t in (o, dq, dk, dv))


def test_a_large_positive_entry_draws_all_attention():
    x, how = make(1, 200, 2, 1, 64, BF, seed=2, bias="bucket", nb=8, reach=20, causal=True)
    how["table"][:, int(how["buckets"][20])] = 1e9
    o, lse = api.attention_forward(x["q"], x["k"], x["v"], **how)
    assert torch.equal(o, x["v"].expand(1, 200, 2, 64))
    dq, dk, dv, dtable = api.attention_backward(x["dout"], x["q"], x["k"], x["v"], o, lse, **how)
    # P = 1 within 2^-6 (see above), then two roundings to bf16
    want = x["dout"].double().sum(2, keepdim=True)
    size = x["dout"].double().abs().sum(2, keepdim=True)
    assert bool(((dv.double() - want).abs() <= (2.0 ** -6 + 2.0 ** -7) * size).all())
    assert all(bool(torch.isfinite(t.float()).all()) for t in (dq, dk, dtable))
