"""The longest sequences, 2^20 tokens of packed short documents: the same values as
the documents in a batch, in 64 bits.  With a table that reaches 512 tokens the
backward pass of width 128 does not fit the tensor-core kernels' shared memory
and runs on the CUDA cores; every other case here runs on the tensor cores."""
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


@pytest.mark.parametrize("D,reach", [(64, 512), (128, 512), (128, 60)])
def test_a_million_tokens_of_short_documents(D, reach):
    L, size, live = 1 << 20, 128, 100               # documents of 100 tokens and 28 of padding
    g = torch.Generator(device="cuda").manual_seed(D + reach)
    q, k, v, dout = (torch.randn(1, L, 1, D, device="cuda", generator=g).to(BF) for _ in range(4))
    at = torch.arange(L, device="cuda")
    ids = torch.where(at % size < live, at // size, -1).int().view(1, L)
    how = {"causal": True, "table": torch.randn(1, 8, device="cuda", generator=g).to(BF),
           "buckets": api.relative_buckets(8, reach, False)}
    o, lse = api.attention_forward(q, k, v, documents=ids, **how)
    dq, dk, dv, dtable = api.attention_backward(dout, q, k, v, o, lse, documents=ids, **how)
    api.attention_error()

    def batch(t):
        return t.view(L // size, size, 1, D)

    ref, err = R.attention(batch(q), batch(k), batch(v), batch(dout), documents=ids.view(L // size, size), **how)
    got = {"o": batch(o), "lse": lse.view(L // size, 1, size), "dq": batch(dq), "dk": batch(dk), "dv": batch(dv),
           "dtable": dtable}
    for name, want in ref.items():
        x = got[name].double()
        ok = ((x - want).abs() <= err[name] + 1e-30) | (torch.isinf(want) & (x == want))
        assert bool(ok.all()), (name, int((~ok).sum()))
