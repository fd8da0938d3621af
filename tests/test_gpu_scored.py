"""Attention with modified scores on the GPU, forward and backward, against the
plain 64-bit implementation with elementwise bounds derived there; strides,
streams, padding that holds NaN, capture and determinism."""
import numpy as np
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


def make(B, L, H, KV, D, dtype, seed=0, bias="none", nb=8, reach=20, causal=False, cap=0.0, docs="none", prefix=False,
         scale=None):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*s):
        return torch.randn(*s, device="cuda", generator=g).to(dtype)

    x = {"q": rnd(B, L, H, D), "k": rnd(B, L, KV, D), "v": rnd(B, L, KV, D), "dout": rnd(B, L, H, D)}
    how = {"causal": causal, "softcap": cap, "scale": scale}
    if bias == "distance":
        how["slopes"] = torch.rand(H, device="cuda", generator=g)
    if bias == "bucket":
        how["table"] = rnd(H, nb)
        how["buckets"] = api.relative_buckets(nb, reach, not causal)
    r = np.random.default_rng(seed)
    if docs != "none":
        ids = np.full((B, L), -1, np.int32)
        for b in range(B):
            if docs == "padded":
                ids[b, : r.integers(0, L + 1)] = 3          # a sequence may be all padding
            elif docs == "packed":
                cuts = np.sort(r.integers(0, L + 1, 5))
                ids[b] = np.searchsorted(cuts, np.arange(L), side="right")
                ids[b, cuts[-1]:] = -1
            else:                                           # ids in no order, padding anywhere
                ids[b] = r.integers(-1, 3, L)
        how["documents"] = torch.from_numpy(ids).cuda()
    if prefix:
        how["prefix"] = torch.from_numpy(r.integers(0, L + 3, B).astype(np.int32)).cuda()
    return x, how


def check(x, how, grads=None, out=None):
    ref, err = R.attention(x["q"], x["k"], x["v"], x["dout"], **how)
    o, lse = api.attention_forward(x["q"], x["k"], x["v"], out=out, **how)
    dq, dk, dv, dtable = api.attention_backward(x["dout"], x["q"], x["k"], x["v"], o, lse, grads=grads, **how)
    api.attention_error()
    got = {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv, "dtable": dtable}
    for name, want in ref.items():
        g = got[name].double()
        same = torch.isinf(want) & (g == want)
        bad = ~(same | ((g - want).abs() <= err[name] + 1e-30))
        worst = float(((g - want).abs() / (err[name] + 1e-30))[~same].max()) if bool((~same).any()) else 0.0
        assert not bool(bad.any()), f"{name}: {int(bad.sum())} of {bad.numel()} outside, worst {worst:.3g} x the bound"
    return got


LENGTHS = [1, 2, 17, 63, 64, 65, 127, 128, 129, 200, 300]


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 32)])
@pytest.mark.parametrize("L", LENGTHS)
def test_lengths(L, dtype, D):
    check(*make(2, L, 4, 2, D, dtype, seed=L, bias="bucket", docs="packed"))
    check(*make(1, L, 2, 2, D, dtype, seed=L + 1, bias="distance", causal=True, cap=15.0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [1, 8, 33, 40, 48, 64, 72, 96, 120, 128])
def test_head_widths(D, dtype):
    check(*make(2, 150, 2, 1, D, dtype, seed=D, bias="bucket", causal=True))


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 48)])
@pytest.mark.parametrize("bias", ["none", "distance", "bucket"])
@pytest.mark.parametrize("cap", [0.0, 10.0])
@pytest.mark.parametrize("causal,docs,prefix", [(False, "none", False), (True, "none", False), (True, "none", True),
                                                (False, "padded", False), (True, "packed", False),
                                                (True, "mixed", True), (False, "mixed", False)])
def test_masks_and_biases(dtype, D, bias, cap, causal, docs, prefix):
    check(*make(2, 290, 4, 2, D, dtype, seed=5, bias=bias, cap=cap, causal=causal, docs=docs, prefix=prefix))


@pytest.mark.parametrize("H,KV", [(1, 1), (8, 1), (6, 2), (5, 5)])
def test_head_groups(H, KV):
    check(*make(2, 200, H, KV, 64, BF, seed=H, bias="bucket", causal=True))
    check(*make(2, 100, H, KV, 32, F32, seed=H, bias="bucket", causal=True))


@pytest.mark.parametrize("nb,reach", [(8, 8), (32, 128), (64, 512), (128, 512)])
@pytest.mark.parametrize("causal", [False, True])
def test_bucket_maps(nb, reach, causal):
    check(*make(1, 1100, 2, 1, 64, BF, seed=nb, bias="bucket", nb=nb, reach=reach, causal=causal))
    x, how = make(2, 257, 2, 2, 64, BF, seed=nb, bias="bucket", nb=nb, reach=reach)
    how["buckets"] = np.random.default_rng(nb).integers(0, nb, 2 * reach + 1).astype(np.uint8)      # any map
    check(x, how)
    check(*make(2, 257, 2, 2, 16, F32, seed=nb, bias="bucket", nb=nb, reach=reach, causal=causal))


def test_longer_sequences():
    check(*make(1, 2100, 2, 1, 128, BF, seed=1, causal=True, cap=30.0, docs="packed"))
    check(*make(1, 1900, 2, 1, 64, BF, seed=2, bias="distance", causal=True, prefix=True))
    check(*make(1, 1000, 2, 1, 64, F32, seed=3, bias="bucket", causal=True))


@pytest.mark.parametrize("dtype,D", [(F32, 32), (F32, 72), (BF, 20), (BF, 64)])
@pytest.mark.parametrize("B,causal", [(1, False), (7, True), (16, False), (24, True)])
def test_small_and_full_grids(B, causal, dtype, D):
    """Few tiles, which several blocks may share, and more tiles than the GPU holds at once."""
    check(*make(B, 330, 6, 3, D, dtype, seed=B, bias="bucket", causal=causal, docs="padded"))


@pytest.mark.parametrize("H,KV,D", [(2, 1, 64), (4, 1, 128), (3, 1, 40), (2, 2, 128)])
@pytest.mark.parametrize("docs,bias", [("none", "none"), ("packed", "bucket"), ("mixed", "distance")])
def test_key_tiles_shared_by_clusters(docs, bias, H, KV, D):
    """Long sequences with few key heads; documents leave some of a cluster's blocks without work."""
    for causal in (False, True):
        check(*make(1, 1100, H, KV, D, BF, seed=H + D, bias=bias, causal=causal, docs=docs))


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
def test_largest_clusters(dtype, D):
    """One head, long enough for clusters of eight blocks."""
    check(*make(1, 4200, 1, 1, D, dtype, seed=D, bias="bucket", docs="packed"))
    check(*make(1, 2300, 3, 1, D, dtype, seed=D, cap=20.0, causal=True, prefix=True))


def test_large_scores():
    """Scores far apart, so that the running maximum moves by more than any threshold."""
    for dtype, D in ((BF, 64), (BF, 128), (F32, 64)):
        x, how = make(1, 700, 2, 2, D, dtype, seed=9, scale=1.0)
        x["k"] = (x["k"].float() * torch.linspace(0.1, 1.5, 700, device="cuda")[None, :, None, None]).to(dtype)
        check(x, how)


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (BF, 36), (F32, 64)])
def test_padding_may_hold_nan_and_infinity(dtype, D):
    x, how = make(3, 300, 4, 2, D, dtype, seed=4, bias="bucket", docs="mixed", causal=True)
    how["documents"][2] = -1                       # a whole sequence of padding
    for i, t in enumerate(x.values()):
        t[how["documents"] < 0] = [float("nan"), float("inf"), float("-inf"), float("nan")][i]
    got = check(x, how)
    pad = how["documents"] < 0
    assert bool((got["o"][pad] == 0).all()) and bool((got["dq"][pad] == 0).all())
    assert bool(torch.isinf(got["lse"].permute(0, 2, 1)[pad]).all())


def test_strides_of_inputs_and_outputs():
    B, L, H, KV, D = 2, 150, 4, 2, 64
    x, how = make(B, L, H, KV, D, BF, seed=6, bias="bucket")
    qkv = torch.cat([x["q"], x["k"], x["v"]], 2)                        # one projection
    dqkv = torch.full_like(qkv, float("nan"))
    parts = (qkv[:, :, :H], qkv[:, :, H:H + KV], qkv[:, :, H + KV:])
    y = dict(x, q=parts[0], k=parts[1], v=parts[2])
    check(y, how, grads=(dqkv[:, :, :H], dqkv[:, :, H:H + KV], dqkv[:, :, H + KV:]))
    assert not bool(torch.isnan(dqkv).any())
    # [B, H, L, D] in memory, for inputs and outputs
    y = {n: t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for n, t in x.items()}
    out = torch.empty(B, H, L, D, dtype=BF, device="cuda").permute(0, 2, 1, 3)
    check(y, how, out=out)
    # an odd offset and odd strides (no 16-byte rows)
    wide = torch.zeros(B, L, H, D + 3, dtype=BF, device="cuda")
    wide[..., 1:D + 1] = x["q"]
    check(dict(x, q=wide[..., 1:D + 1]), how)
    # one sequence of keys for the whole batch, one gradient for every token
    check(dict(x, k=x["k"][:1].expand(B, L, KV, D), dout=x["dout"][:, :1].expand(B, L, H, D)), how)


def test_gradient_expanded_from_a_scalar():
    x, how = make(2, 40, 2, 2, 64, BF, seed=7)
    x["dout"] = torch.ones((), dtype=BF, device="cuda").expand(2, 40, 2, 64)
    check(x, how)


def test_offsets_beyond_32_bits():
    """Tokens 2^23 elements apart: byte offsets up to 5 GB."""
    L, step = 300, 1 << 23
    big = torch.empty(L * step, dtype=BF, device="cuda")
    x, how = make(1, L, 1, 1, 64, BF, seed=8, causal=True)
    at = 0
    for n in ("q", "k", "v", "dout"):
        t = big.as_strided((1, L, 1, 64), (L * step, step, 64, 1), at)
        t.copy_(x[n])
        x[n], at = t, at + 64
    out = big.as_strided((1, L, 1, 64), (L * step, step, 64, 1), at)
    check(x, how, out=out)


def test_equal_calls_give_equal_bits():
    for dtype, D in ((BF, 64), (BF, 128), (F32, 32)):
        x, how = make(2, 500, 4, 1, D, dtype, seed=10, bias="bucket", cap=20.0, docs="packed")
        runs = [check(x, how) for _ in range(2)]
        for n in runs[0]:
            assert torch.equal(runs[0][n], runs[1][n]), n


def test_another_stream_and_capture():
    x, how = make(2, 200, 4, 2, 64, BF, seed=11, bias="bucket", docs="packed")
    ref, err = R.attention(x["q"], x["k"], x["v"], x["dout"], **how)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o, lse = api.attention_forward(x["q"], x["k"], x["v"], stream=s.cuda_stream, **how)
    s.synchronize()
    assert bool(((o.double() - ref["o"]).abs() <= err["o"]).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2, lse2 = api.attention_forward(x["q"], x["k"], x["v"], **how)
        g2 = api.attention_backward(x["dout"], x["q"], x["k"], x["v"], o2, lse2, **how)
    x["q"].copy_(torch.randn_like(x["q"]))
    graph.replay()
    torch.cuda.synchronize()
    ref, err = R.attention(x["q"], x["k"], x["v"], x["dout"], **how)
    for name, got in zip(("o", "dq", "dk", "dv", "dtable"), (o2, *g2)):
        assert bool(((got.double() - ref[name]).abs() <= err[name]).all()), name


def test_zero_lengths():
    for B, L in ((0, 16), (2, 0)):
        q = torch.empty(B, L, 2, 64, dtype=BF, device="cuda")
        table = torch.ones(2, 8, dtype=BF, device="cuda")
        how = {"table": table, "buckets": api.relative_buckets(8, 20)}
        o, lse = api.attention_forward(q, q, q, **how)
        dq, dk, dv, dtable = api.attention_backward(q, q, q, q, o, lse, **how)
        assert o.shape == q.shape and dq.shape == q.shape and bool((dtable == 0).all())


@pytest.mark.parametrize("cap,bias", [(0.0, "bucket"), (5.0, "bucket"), (5.0, "distance")])
def test_gradients_against_differences(cap, bias):
    """<gradient, direction> against central differences of the 64-bit
    forward's loss sum(dout * o) along that direction, step 1e-4: truncation
    ~1e-8 of the third derivative, rounding ~1e-12."""
    x, how = make(2, 70, 4, 2, 32, F32, seed=12, cap=cap, bias=bias, causal=True, docs="packed")
    o, lse = api.attention_forward(x["q"], x["k"], x["v"], **how)
    dq, dk, dv, dtable = api.attention_backward(x["dout"], x["q"], x["k"], x["v"], o, lse, **how)
    g = torch.Generator(device="cuda").manual_seed(1)
    live = (how["documents"] >= 0)[:, :, None, None]
    for name, grad in (("q", dq), ("k", dk), ("v", dv)) + ((("table", dtable),) if bias == "bucket" else ()):
        at = x[name] if name != "table" else how["table"]
        d = torch.randn(at.shape, device="cuda", generator=g, dtype=torch.float64)

        def loss(t):
            y = {n: x[n].double() for n in ("q", "k", "v")}
            h = dict(how)
            if name == "table":
                h["table"] = at.double() + t * d
            else:
                y[name] = y[name] + t * d
            return float((R64(y, h) * torch.where(live, x["dout"].double(), 0.0)).sum())

        diff = (loss(1e-4) - loss(-1e-4)) / 2e-4
        got = float((grad.double() * d).sum())
        size = float((grad.double().abs() * d.abs()).sum())
        assert abs(got - diff) <= 1e-6 * size + 1e-6, (name, got, diff)


def R64(y, how):
    R.ROUND.setdefault(torch.float64, 2.0 ** -53)
    return R.attention(y["q"], y["k"], y["v"], **how)[0]["o"]


def test_bad_arguments_are_refused():
    x, how = make(1, 32, 4, 2, 64, BF)
    q, k, v = x["q"], x["k"], x["v"]
    table, buckets = torch.zeros(4, 8, dtype=BF, device="cuda"), api.relative_buckets(8, 20)
    fwd = api.attention_forward
    with pytest.raises(ValueError):
        fwd(q.half(), k.half(), v.half())
    with pytest.raises(ValueError):
        fwd(q, k, v[:, :16])
    with pytest.raises(ValueError):
        fwd(q, k.float(), v)
    with pytest.raises(ValueError):
        fwd(q.cpu(), k.cpu(), v.cpu())
    with pytest.raises(ValueError):
        fwd(q.permute(0, 1, 3, 2), k, v)
    with pytest.raises(ValueError):
        fwd(q, k, v, table=table)
    with pytest.raises(ValueError):
        fwd(q, k, v, table=table.float(), buckets=buckets)
    with pytest.raises(ValueError):
        fwd(q, k, v, documents=torch.zeros(1, 32, dtype=torch.int64, device="cuda"))
    with pytest.raises(api.FedOptimaError, match="below buckets"):
        fwd(q, k, v, table=table[:, :7].contiguous(), buckets=buckets)
    with pytest.raises(api.FedOptimaError, match="prefix"):
        fwd(q, k, v, prefix=torch.zeros(1, dtype=torch.int32, device="cuda"))
    with pytest.raises(api.FedOptimaError, match="one of slopes and table"):
        fwd(q, k, v, table=table, buckets=buckets, slopes=torch.zeros(4, device="cuda"))
    with pytest.raises(api.FedOptimaError, match="softcap"):
        fwd(q, k, v, softcap=-1.0)
    with pytest.raises(api.FedOptimaError, match="scale"):
        fwd(q, k, v, scale=float("nan"))
    with pytest.raises(api.FedOptimaError, match="multiple"):
        fwd(q[:, :, :3], k, v)
    with pytest.raises(api.FedOptimaError, match="head_dim"):
        w = torch.zeros(1, 8, 1, 136, dtype=BF, device="cuda")
        fwd(w, w, w)
    with pytest.raises(api.FedOptimaError, match="strides"):
        fwd(q, k, v, out=torch.zeros(1, 1, 4, 64, dtype=BF, device="cuda").expand(1, 32, 4, 64))
