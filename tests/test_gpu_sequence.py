"""Devices training transformer blocks with scored attention and dropout, and
feeding the server: the local loss falls, the server trains on the uploads, and
the blocks' gradients agree with torch's in 64 bits."""
import math

import numpy as np
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


def test_devices_feed_the_server():
    from paper_2504_13850_gb300 import sequence
    local, server = sequence.run(events=24, devices=2, vocab=500)
    assert len(local) == len(server) == 24 and np.all(np.isfinite(local)) and np.all(np.isfinite(server))
    # two labels per device's one batch, seen twelve times: from about ln 2 down
    assert abs(np.mean(local[:2]) - math.log(2)) < 0.35
    assert np.mean(local[-2:]) < 0.5 * np.mean(local[:2])


def test_block_gradients_match_torch():
    """Attention, its output projection and the dropout around the residual, as
    the device chains them, against the same chain in 64 bits.  Bound: each of
    the five bf16 tensors on the way (o, its projection, y and their gradients)
    is off by 2^-8 relative per element; errors of independent elements add in
    the 2-norm, so 5 * 2^-8 covers every gradient normwise."""
    from paper_2504_13850_gb300 import sequence as S
    B, L, H, D, p, seed, call = 3, 100, 4, 64, 0.2, 9, 5
    g = torch.Generator(device="cuda").manual_seed(2)

    def leaf(*shape):
        return torch.randn(*shape, device="cuda", generator=g).bfloat16().requires_grad_()

    qkv, table, w, x = leaf(B, L, 3, H, D), leaf(H, S.BUCKETS), leaf(H * D, H * D), leaf(B, L, H * D)
    buckets = api.relative_buckets(S.BUCKETS, S.REACH)
    docs = torch.where(torch.arange(L, device="cuda") < torch.tensor([[100], [57], [8]], device="cuda"), 0, -1).int()
    o = S.PackedAttention.apply(qkv, table, buckets, docs)
    y = S.ResidualDropout.apply(o.reshape(B, L, -1) @ (w / 16), x, p, seed, call)
    dy = torch.randn(B, L, H * D, device="cuda", generator=g).bfloat16()
    y.backward(dy)

    ref = [t.detach().double().requires_grad_() for t in (qkv, table, w, x)]
    q, k, v = ref[0].permute(2, 0, 3, 1, 4)
    at = torch.arange(L, device="cuda")
    which = torch.from_numpy(buckets.astype(np.int64)).cuda()[(at[None, :] - at[:, None]).clamp(-S.REACH, S.REACH) + S.REACH]
    z = q @ k.mT / 8 + ref[1][:, which]
    ok = ((docs[:, :, None] == docs[:, None, :]) & (docs >= 0)[:, :, None])[:, None]
    P = torch.nan_to_num(torch.softmax(z.masked_fill(~ok, float("-inf")), -1))
    keep, scale = R.dropout_mask(x.numel(), p, seed, call)
    keep = torch.from_numpy(keep).cuda().view(x.shape)
    Y = ref[3] + torch.where(keep, ((P @ v).permute(0, 2, 1, 3).reshape(B, L, -1) @ (ref[2] / 16)) * scale, 0.0)
    Y.backward(dy.double())
    for name, a, b in zip(("y", "qkv", "table", "w", "x"), (y, qkv.grad, table.grad, w.grad, x.grad),
                          (Y, *(t.grad for t in ref))):
        err = float((a.detach().double() - b.detach()).norm() / b.detach().norm())
        assert err <= 5 * 2.0 ** -8, (name, err)
