"""Embedding lookup and its gradient on the GPU against 64 bits, element by
element: types, odd widths, padding, ids that fill the batch, strides, offsets
beyond 32 bits, capture, other streams.

Bounds: a lookup is one fp32 product (2^-24) and one rounding; a gradient of n
tokens at most n - 1 fp32 additions, whose order does not matter for the bound
n 2^-24 sum |dout|, a product and a rounding."""
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TYPES = [(F32, F32), (F32, BF), (BF, BF)]             # table, activations
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


def make(T, V, D, table, dtype, seed=0, ids=None, padded=0.2, id_type=torch.int32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if ids is None:
        ids = (torch.pow(float(V + 1), torch.rand(T, device="cuda", generator=g, dtype=torch.float64)).long() - 1).clamp(0, V - 1)
        ids[torch.rand(T, device="cuda", generator=g) < padded] = -1
    w = torch.randn(V, D, device="cuda", generator=g).to(table)
    dout = torch.randn(*ids.shape, D, device="cuda", generator=g).to(dtype)
    return ids.to(id_type), w, dout


def lookup_agrees(got, ids, w, scale):
    V = w.shape[0]
    fine = ((ids >= 0) & (ids < V))[..., None]
    want = torch.where(fine, w.double()[ids.long().clamp(0, V - 1)] * scale, 0.0)
    return bool(((got.double() - want).abs() <= (R.ROUND[got.dtype] + U) * want.abs()).all())


def grad_want(dout, ids, V, scale):
    """(dtable, bound without its rounding) in 64 bits."""
    D = dout.shape[-1]
    flat, d = ids.reshape(-1).long(), dout.reshape(-1, D).double()
    keep = (flat >= 0) & (flat < V)
    flat, d = flat[keep], d[keep]
    want = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, flat, d) * scale
    size = torch.zeros_like(want).index_add_(0, flat, d.abs()) * abs(scale)
    n = torch.bincount(flat, minlength=V)[:, None]
    return want, (n + 1) * U * size


def grad_agrees(got, dout, ids, V, scale, before=None):
    want, bound = grad_want(dout, ids, V, scale)
    if before is not None:
        bound = bound + U * before.double().abs()
        want = want + before.double()
    return bool(((got.double() - want).abs() <= bound + (R.ROUND[got.dtype] + U) * (want.abs() + bound)).all())


@pytest.mark.parametrize("table,dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 50, 8), (2, 3, 7), (31, 10, 64), (32, 512, 256), (33, 511, 257), (64, 513, 512),
                                   (1000, 7, 40), (4096, 30522, 512), (5000, 1000, 777), (20000, 262144, 24), (300, 100, 2056),
                                   (16384, 300, 16), (16385, 300, 16), (5000, 1 << 20, 8), (16384, 40000, 8)])
def test_values_and_gradients(table, dtype, T, V, D):
    for k, id_type in enumerate((torch.int32, torch.int64)):
        ids, w, dout = make(T, V, D, table, dtype, seed=k, id_type=id_type)
        assert lookup_agrees(api.embedding(ids, w, scale=D ** 0.5, dtype=dtype), ids, w, float(torch.tensor(D ** 0.5)))
        got = api.embedding_grad(dout, ids, V, scale=D ** 0.5, dtype=table)
        assert grad_agrees(got, dout, ids, V, float(torch.tensor(D ** 0.5)))


@pytest.mark.parametrize("D", [16, 19])
@pytest.mark.parametrize("case", ["one id", "two ids", "runs of 32", "runs of 33", "all padding", "ends", "descending", "bad ids"])
def test_ids_that_fill_the_batch(case, D):
    """Rows whose tokens fill pieces, begin and end on their edges, or miss."""
    T, V = 3000, 700
    at = torch.arange(T, device="cuda")
    ids = {"one id": torch.full((T,), 5, device="cuda"), "two ids": torch.where(at < 1471, V - 1, 0), "runs of 32": at // 32,
           "runs of 33": at // 33, "all padding": torch.full((T,), -1, device="cuda"),
           "ends": torch.where(at % 2 == 0, 0, V - 1), "descending": (T - 1 - at) * V // T,
           "bad ids": torch.where(at % 3 == 0, V + at, torch.where(at % 3 == 1, -at - 1, at % V))}[case]
    ids, w, dout = make(T, V, D, F32, F32, ids=ids, id_type=torch.int64)
    assert lookup_agrees(api.embedding(ids, w), ids, w, 1.0)
    assert grad_agrees(api.embedding_grad(dout, ids, V), dout, ids, V, 1.0)


def test_padding_holds_anything():
    ids, w, dout = make(500, 40, 33, F32, F32, padded=0.5)
    clean = api.embedding_grad(dout, ids, 40)
    dout[ids < 0] = float("nan")
    assert torch.equal(api.embedding_grad(dout, ids, 40), clean)
    w[7] = float("inf")
    out = api.embedding(ids, w, scale=0.0)
    assert bool((out[ids < 0] == 0).all()) and bool(out[ids == 7].isnan().all())


@pytest.mark.parametrize("table,dtype", TYPES)
@pytest.mark.parametrize("D,pad,skip", [(64, 8, 0), (64, 3, 1), (13, 5, 2)])
def test_strides_and_shapes(table, dtype, D, pad, skip):
    ids, w, _ = make(90, 50, D, table, dtype)
    big = torch.randn(90, D + pad, device="cuda").to(dtype)
    before, out = big.clone(), big[:, skip:skip + D]
    y = api.embedding(ids, w, dtype=dtype, out=out)
    assert lookup_agrees(y, ids, w, 1.0)
    before[:, skip:skip + D] = y
    assert torch.equal(before, big)                     # nothing between the rows was written
    assert grad_agrees(api.embedding_grad(out, ids, 50, dtype=table), out, ids, 50, 1.0)
    shaped = ids.view(3, 5, 6)
    assert torch.equal(api.embedding(shaped, w, dtype=dtype), y.reshape(3, 5, 6, D))
    for g in (torch.randn(D, device="cuda").to(dtype).expand(3, 5, 6, D), torch.randn(3, 5, 6, 1, device="cuda").to(dtype).expand(3, 5, 6, D),
              torch.randn(1, D, device="cuda").to(dtype).expand(90, D)):
        i = shaped if g.dim() == 4 else ids
        assert grad_agrees(api.embedding_grad(g, i, 50, dtype=table), g, i, 50, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("D", [32, 21])
def test_accumulation(dtype, D):
    ids, w, dout = make(2000, 100, D, dtype, dtype)
    ids[ids == 17] = 16                                  # a row without a token keeps its bits
    before = torch.randn(100, D, device="cuda").to(dtype)
    got = api.embedding_grad(dout, ids, 100, scale=0.5, out=before.clone(), accumulate=True)
    assert grad_agrees(got, dout, ids, 100, 0.5, before) and torch.equal(got[17], before[17])
    over = torch.full((100, D), float("nan"), device="cuda", dtype=dtype)
    assert grad_agrees(api.embedding_grad(dout, ids, 100, out=over), dout, ids, 100, 1.0)


def test_no_tokens():
    ids = torch.empty(0, 4, device="cuda", dtype=torch.int32)
    w = torch.randn(5, 8, device="cuda")
    assert api.embedding(ids, w).shape == (0, 4, 8)
    assert bool((api.embedding_grad(torch.empty(0, 4, 8, device="cuda"), ids, 5) == 0).all())
    assert torch.equal(api.embedding_grad(torch.empty(0, 4, 8, device="cuda"), ids, 5, out=w.clone(), accumulate=True), w)


def test_gradient_by_differences():
    """The lookup is linear in the table: its difference along d is lookup(d)."""
    ids, w, dout = make(777, 60, 40, F32, F32)
    d = torch.randn_like(w)
    step = (api.embedding(ids, w + d, scale=3.0).double() - api.embedding(ids, w - d, scale=3.0).double()) / 2
    got = (api.embedding_grad(dout, ids, 60, scale=3.0).double() * d.double()).sum()
    # fp32 roundings of the inputs w +- d, of both products, and of the gradient's sums (at most 777 terms)
    size = (dout.double().abs() * api.embedding(ids, w.abs() + d.abs(), scale=3.0).double()).sum()
    assert abs(float((step * dout.double()).sum() - got)) <= 800 * U * float(size)


def test_equal_calls_give_equal_bits_and_tokens_order_is_kept():
    ids, w, dout = make(6000, 50, 128, BF, BF)
    first = api.embedding_grad(dout, ids, 50)
    for _ in range(3):
        assert torch.equal(api.embedding_grad(dout, ids, 50), first)


def test_sorts_give_equal_bits():
    """8192 tokens are sorted by one block where an id and a token's number fit 32
    bits, else by launches: the same order, so the same sums."""
    ids, w, dout = make(8192, 300, 24, F32, F32)
    small, large = api.embedding_grad(dout, ids, 300), api.embedding_grad(dout, ids, 1 << 19)
    assert torch.equal(large[:300], small) and float(large[300:].abs().max()) == 0


@pytest.mark.parametrize("table,dtype", TYPES)
@pytest.mark.parametrize("T,V,D", [(8192, 3000, 16), (8193, 3000, 16), (16385, 1, 8), (17000, 40, 9), (24576, 511, 32), (40000, 512, 8), (65536, 100000, 40), (131071, 3000, 16),
                                   (131072, 30522, 8), (131073, 30522, 8), (300000, 700, 17), (300, 1 << 26, 1), (1, (1 << 27) + 1, 2)])
def test_many_tokens_and_rows(table, dtype, T, V, D):
    """More tokens, or larger ids, than one block sorts."""
    ids, w, dout = make(T, V, D, table, dtype, id_type=torch.int64 if V % 2 else torch.int32)
    over = torch.full((V, D), float("nan"), device="cuda", dtype=table)
    got = api.embedding_grad(dout, ids, V, scale=0.5, out=over)
    if V > 1 << 20:                                      # few rows have tokens: only those in 64 bits
        rows, back = ids.clamp(min=0).long().unique(return_inverse=True)
        part = torch.where(ids < 0, -1, back)
        assert grad_agrees(got[rows], dout, part, len(rows), 0.5)
        got[rows] = 0
        assert float(got.abs().max()) == 0
        return
    assert grad_agrees(got, dout, ids, V, 0.5)
    before = torch.randn(V, D, device="cuda").to(table)
    got = api.embedding_grad(dout, ids, V, scale=0.5, out=before.clone(), accumulate=True)
    assert grad_agrees(got, dout, ids, V, 0.5, before)


@pytest.mark.parametrize("T", [20000, 140000])
@pytest.mark.parametrize("case", ["one id", "runs of 33", "all padding", "ends", "descending", "bad ids"])
def test_ids_that_fill_large_batches(case, T):
    V, at = 700, torch.arange(T, device="cuda")
    ids = {"one id": torch.full((T,), 5, device="cuda"), "runs of 33": at // 33, "all padding": torch.full((T,), -1, device="cuda"),
           "ends": torch.where(at % 2 == 0, 0, V - 1), "descending": (T - 1 - at) * V // T,
           "bad ids": torch.where(at % 3 == 0, V + at, torch.where(at % 3 == 1, -at - 1, at % V))}[case]
    ids, w, dout = make(T, V, 24, F32, F32, ids=ids, id_type=torch.int64)
    assert grad_agrees(api.embedding_grad(dout, ids, V), dout, ids, V, 1.0)


def test_capture_and_other_streams():
    """Captured and replayed on new inputs, beside calls on two other streams."""
    ids, w, dout = make(3000, 500, 96, F32, BF)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        api.embedding(ids, w, dtype=BF), api.embedding_grad(dout, ids, 500, dtype=F32)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        y = api.embedding(ids, w, dtype=BF)
        d = api.embedding_grad(dout, ids, 500, dtype=F32)
    for seed in (5, 6):
        i2, w2, d2 = make(3000, 500, 96, F32, BF, seed=seed)
        ids.copy_(i2), w.copy_(w2), dout.copy_(d2)
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        graph.replay()
        e = api.embedding_grad(dout, ids, 500, dtype=F32, stream=other.cuda_stream)
        torch.cuda.synchronize()
        assert lookup_agrees(y, ids, w, 1.0) and grad_agrees(d, dout, ids, 500, 1.0) and torch.equal(d, e)


def test_offsets_beyond_32_bits():
    V, D = (1 << 20) + 3, 2080                            # 2.2e9 elements
    w = torch.zeros(V, D, device="cuda", dtype=BF)
    w[V - 1], w[0] = 3.0, 1.0
    ids = torch.tensor([V - 1, 0, V - 2, V - 1], device="cuda")
    assert api.embedding(ids, w)[:, -1].tolist() == [3.0, 1.0, 0.0, 3.0]
    w.fill_(float("nan"))
    got = api.embedding_grad(torch.ones(4, D, device="cuda", dtype=BF), ids, V, out=w)
    assert bool((got[V - 1] == 2).all()) and bool((got[0] == 1).all()) and bool((got[V - 2] == 1).all())
    for i in range(0, V, 1 << 17):
        part = got[i:i + (1 << 17)].float().sum(1)
        assert float(part.sum()) == D * sum({0: 1, V - 2: 1, V - 1: 2}.get(j, 0) for j in (0, V - 2, V - 1) if i <= j < i + (1 << 17))


def test_refusals():
    ids, w, dout = make(10, 20, 16, F32, F32)
    for call in (lambda: api.embedding(ids.float(), w), lambda: api.embedding(ids, w.t()), lambda: api.embedding(ids.cpu(), w),
                 lambda: api.embedding(ids, w.half()), lambda: api.embedding(ids, w, out=torch.empty(10, 15, device="cuda")),
                 lambda: api.embedding_grad(dout[:9], ids, 20), lambda: api.embedding_grad(dout, ids, 20, accumulate=True),
                 lambda: api.embedding_grad(dout, ids, 21, out=w), lambda: api.embedding_grad(dout, ids[::2], 20)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(api.FedOptimaError, match="fp32 table"):
        api.embedding(ids, w.bfloat16(), dtype=F32)
    with pytest.raises(api.FedOptimaError, match="stride"):
        api.embedding(ids, w, out=torch.empty(1, 16, device="cuda").expand(10, 16))
