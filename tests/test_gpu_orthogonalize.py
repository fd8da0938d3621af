"""Orthogonalised updates on the GPU against 64 bits.

The bound follows the formula on the 64-bit iterates, in Frobenius norms.  A step
f(X) = X p(X^T X) passes an error on with at most L = max |f'| over the singular
values (a function of singular values that is odd has this Lipschitz constant),
and adds its own: X, A and B are rounded to operands (d = 2^-12 for bf16 matrices,
whose operands are fp16, 2^-22 for fp32 ones, whose operands are pairs), and sums
lose g = 2^-23 of the sum of absolute values per 16 terms (512 for fp32 matrices,
whose sums are moved and added in fp32 then, with 2^-24 each)."""
import math

import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()
    yield
    api.orthogonalize_error()


def sums_loss(dtype, terms):
    if dtype == BF:
        return (terms / 16 + 1) * 2.0 ** -23
    return (min(terms, 512) / 16 + 3) * 2.0 ** -23 + (terms / 512 + 1) * U


def reference(u, dtype, steps=5, coefficients=api.QUINTIC, eps=1e-7):
    """(X, bound of the error's Frobenius norm before the result's rounding)."""
    a, b, c = coefficients
    X = u.double()
    flip = X.shape[0] > X.shape[1]
    X = X.t() if flip else X
    # the norm's fp32 sums and the scaling to the first operand
    n = math.sqrt(float(X.square().sum())) + eps
    X = X / n
    d = 2.0 ** -12 if dtype == BF else 2.0 ** -22
    e = (100 * U) * float(X.norm())
    m, k = X.shape
    for _ in range(steps):
        A = X @ X.t()
        S, F = float(torch.linalg.eigvalsh(A)[-1].clamp(min=0).sqrt()), float(X.norm())
        s = torch.linspace(0, 1.05 * S + 1e-3, 2000, dtype=torch.float64)
        L = float((a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max())
        B = a * torch.eye(m, dtype=X.dtype, device=X.device) + b * A + c * A @ A
        new = B @ X
        gram = d * float(A.norm()) + sums_loss(dtype, k) * float((X.abs() @ X.abs().t()).norm())
        poly = (abs(b) + 2 * abs(c) * S * S) * gram + abs(c) * sums_loss(dtype, m) * float((A.abs() @ A.abs()).norm())
        poly += (d + 4 * U) * float(B.norm()) + 4 * U * (abs(b) * float(A.norm()) + abs(c) * float((A @ A).norm()))
        e = L * (e + d * F) + poly * S + sums_loss(dtype, m) * float((B.abs() @ X.abs()).norm())
        X = new
    return (X.t() if flip else X), e


def agrees(got, u, **how):
    want, e = reference(u, got.dtype, **how)
    off = float((got.double() - want).norm())
    return off <= 1.05 * e + R.ROUND[got.dtype] * float(want.norm())


def make(rows, cols, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = min(rows, cols, 5)
    u = torch.randn(rows, k, device="cuda", generator=g) * 0.5 ** torch.arange(k, device="cuda")
    return (u @ torch.randn(k, cols, device="cuda", generator=g) + 0.2 * torch.randn(rows, cols, device="cuda", generator=g)).to(dtype)


# up to 128 x 2048 in shared memory; above, tiles of pairs, and clusters that share the long sums of few tiles
SHAPES = [(1, 1), (1, 9), (8, 1), (3, 5), (64, 64), (63, 65), (128, 128), (129, 127), (96, 200), (200, 96), (256, 130), (130, 384), (512, 513),
          (1000, 77), (40, 3000), (512, 2048), (1536, 512), (700, 1100), (128, 2048),
          (100, 2049), (1300, 128), (140, 4096), (300, 2500), (1920, 2100)]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_values(dtype, rows, cols):
    u = make(rows, cols, dtype)
    assert agrees(api.orthogonalize(u), u)


@pytest.mark.parametrize("rows,cols", [(2400, 2400), (2600, 2500), (2900, 2900)])
def test_more_tiles_than_pairs(rows, cols):
    """100, 110 and (of X X^T) 78 tiles of 256 x 256 for 76 pairs, some of them
    beyond the matrix's edge by half."""
    u = make(rows, cols, BF)
    assert agrees(api.orthogonalize(u), u)


def test_more_tiles_than_pairs_of_several_matrices():
    """96 tiles of C X.  The second's and third's sums of X X^T are shared by several
    pairs where they have the device to themselves (12 and 20 tiles of 128 columns
    for 76 pairs), and are taken in another order here."""
    us = [make(r, c, BF, seed=k) for k, (r, c) in enumerate([(1500, 1700), (700, 2400), (1300, 1000), (40, 50)])]
    for k, (u, x) in enumerate(zip(us, api.orthogonalize(us))):
        assert agrees(x, u)
        assert k in (1, 2) or torch.equal(x, api.orthogonalize(u))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", [(300, 300), (260, 700), (700, 260)])
def test_places(dtype, rows, cols):
    """One nonzero per row and column: each has a polynomial of its own value,
    and every other element stays zero."""
    n = min(rows, cols)
    g = torch.Generator().manual_seed(1)
    i, j = torch.randperm(rows, generator=g)[:n].cuda(), torch.randperm(cols, generator=g)[:n].cuda()
    u = torch.zeros(rows, cols, device="cuda", dtype=dtype)
    u[i, j] = torch.linspace(0.5, 1.5, n, device="cuda").to(dtype)
    got = api.orthogonalize(u)
    x = u[i, j].double()
    x = x / (x.norm() + 1e-7)
    a, b, c = api.QUINTIC
    e = 100 * U * x
    d = 2.0 ** -12 if dtype == BF else 2.0 ** -22
    for _ in range(5):
        A = x * x
        local = d * (4 * a + 2 * abs(b) * A * 3 + 3 * abs(c) * A * A * 5) * x      # roundings of X, A, B on the way
        e = (a + 3 * b * A + 5 * c * A * A).abs() * e + local + 20 * U * x
        x = x * (a + b * A + c * A * A)
    assert bool(((got[i, j].double() - x).abs() <= 1.1 * e + R.ROUND[dtype] * x.abs()).all())
    got[i, j] = 0
    assert float(got.abs().max()) == 0


@pytest.mark.parametrize("dtype", [F32, BF])
def test_lists_equal_single_calls(dtype):
    """More matrices than one launch holds, of all shapes, and empty ones."""
    us = [make(r, c, dtype, seed=k) for k, (r, c) in enumerate(SHAPES[:12] * 3)]
    us.insert(3, torch.empty(0, 7, device="cuda", dtype=dtype))
    got = api.orthogonalize(us)
    assert len(got) == len(us) == 37 and got[3].shape == (0, 7)
    for u, x in zip(us, got):
        assert torch.equal(x, api.orthogonalize(u))
    assert api.orthogonalize([]) == []


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_other_polynomials(steps):
    u = make(150, 260, F32)
    how = dict(steps=steps, coefficients=(1.875, -1.25, 0.375), eps=1e-3)
    x = api.orthogonalize(u, **how)
    assert agrees(x, u, **how)
    how = dict(steps=steps, coefficients=(1.5, -0.5, 0.0))
    assert agrees(api.orthogonalize(u.t(), **how), u.t().contiguous(), **how)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e30])
def test_magnitudes(dtype, size):
    u = (make(200, 140, F32).double() * size).to(dtype)
    eps = 1e-30 if size < 1 else 1e-7
    x = api.orthogonalize(u, eps=eps)
    assert agrees(x, u.double(), eps=eps) if x.dtype == F32 else agrees(x, u, eps=eps)


def test_zeros_and_not_finite():
    z = torch.zeros(100, 150, device="cuda")
    assert float(api.orthogonalize(z).abs().max()) == 0
    for bad in (float("nan"), float("inf"), -float("inf")):
        u = make(100, 150, F32)
        u[3, 77] = bad
        x, y = api.orthogonalize([u, make(90, 90, F32)])
        assert bool(x.isnan().all()) and agrees(y, make(90, 90, F32))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_strides(dtype):
    big = torch.randn(210, 170, device="cuda").to(dtype)
    u = big[3:203, 5:146]
    want = api.orthogonalize(u.contiguous())
    out = torch.full((200, 150), 7.0, device="cuda", dtype=dtype)
    x = api.orthogonalize(u, out=out[:, 4:145])
    assert torch.equal(x, want) and bool((out[:, :4] == 7).all()) and bool((out[:, 145:] == 7).all())
    t = u.t()                                             # columns along memory: copied
    assert torch.equal(api.orthogonalize(t), api.orthogonalize(t.contiguous()))
    one = torch.randn(1, 90, device="cuda").to(dtype).expand(60, 90)
    assert agrees(api.orthogonalize(one), one)
    w = u.contiguous()
    assert torch.equal(api.orthogonalize(w, out=w), want) and torch.equal(w, want)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_steps(dtype, nesterov):
    """Three steps with momentum and decay, parameters inside wider rows."""
    shapes = [(150, 90), (90, 150), (128, 256), (5, 3)]
    store = [torch.randn(r, c + 3, device="cuda") for r, c in shapes]
    params = [s[:, 1:-2] for s in store]
    momenta = [torch.zeros(r, c, device="cuda") for r, c in shapes]
    P, M = [p.double() for p in params], [m.double() for m in momenta]
    edges = [s[:, [0, -2, -1]].clone() for s in store]
    e = [0.0] * len(shapes)
    for k in range(3):
        grads = [make(r, c, dtype, seed=10 * k + i) for i, (r, c) in enumerate(shapes)]
        before = [m.clone() for m in momenta]
        api.muon_step(params, grads, momenta, lr=0.1, momentum=0.9, nesterov=nesterov, weight_decay=0.2)
        for i, (r, c) in enumerate(shapes):
            m = torch.addcmul(grads[i].float(), before[i], torch.full((), 0.9, device="cuda"))
            assert bool(((momenta[i] - m).abs() <= 2 * U * (m.abs() + grads[i].float().abs() + before[i].abs())).all())
            u = grads[i].double() + float(torch.tensor(0.9)) * momenta[i].double() if nesterov else momenta[i].double()
            x, bound = reference(u, dtype)
            scale = max(1.0, r / c) ** 0.5
            P[i] = P[i] * (1 - 0.1 * 0.2) - 0.1 * scale * x
            # U's own fp32 rounding passes through the five steps like the first operand's
            e[i] += 0.1 * scale * (1.05 * bound + 2000 * U) + 4 * U * float(P[i].norm())
            assert float((params[i].double() - P[i]).norm()) <= e[i], (k, i)
    assert all(torch.equal(s[:, [0, -2, -1]], b) for s, b in zip(store, edges))


def test_singular_values():
    """Every direction of a full-rank update ends in the band that the five steps
    reach from its own start."""
    u = make(256, 400, F32)
    s0 = torch.linalg.svdvals(u.double())
    s0 = s0 / (u.double().norm() + 1e-7)
    a, b, c = api.QUINTIC
    for _ in range(5):
        s0 = s0 * (a + b * s0 ** 2 + c * s0 ** 4)
    got = torch.linalg.svdvals(api.orthogonalize(u).double())
    assert float((got.sort()[0] - s0.sort()[0]).abs().max()) <= reference(u, F32)[1] + U * float(s0.norm())
    assert 0.3 < float(got.min()) and float(got.max()) < 1.3


def test_equal_calls_give_equal_bits():
    for dtype in (F32, BF):
        us = [make(512, 768, dtype), make(900, 300, dtype)]
        first = api.orthogonalize(us)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, api.orthogonalize(us)))


def test_capture_and_other_streams():
    us = [make(300, 200, F32), make(128, 640, F32)]
    api.orthogonalize(us)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        xs = api.orthogonalize(us)
    for seed in (3, 4):
        for u in us:
            u.copy_(make(*u.shape, F32, seed=seed))
        torch.cuda.synchronize()
        graph.replay()
        ys = api.orthogonalize(us, stream=other.cuda_stream)
        torch.cuda.synchronize()
        assert all(agrees(x, u) and torch.equal(x, y) for u, x, y in zip(us, xs, ys))


def test_refusals():
    u = make(20, 30, F32)
    for call in (lambda: api.orthogonalize(u[0]), lambda: api.orthogonalize(u.half()), lambda: api.orthogonalize(u.cpu()),
                 lambda: api.orthogonalize([u, u.bfloat16()]), lambda: api.orthogonalize(u, out=u[:10]),
                 lambda: api.orthogonalize([u], out=[u, u]), lambda: api.muon_step([u], [u], [u.bfloat16()], 0.1),
                 lambda: api.muon_step([u.bfloat16()], [u], [u], 0.1), lambda: api.muon_step([u], [u, u], [u], 0.1)):
        with pytest.raises(ValueError):
            call()
    for how, what in ((dict(steps=0), "steps"), (dict(steps=65), "steps"), (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"),
                      (dict(coefficients=(1.0, float("nan"), 0.0)), "coefficients"), (dict(coefficients=(1e3, 0.0, 0.0)), "coefficients")):
        with pytest.raises(api.FedOptimaError, match=what):
            api.orthogonalize(u, **how)
    with pytest.raises(api.FedOptimaError, match="stride"):
        api.orthogonalize(u, out=torch.empty(1, 30, device="cuda").expand(20, 30))
    with pytest.raises(api.FedOptimaError, match="momentum"):
        api.muon_step([u], [u], [u.clone()], 0.1, momentum=1.5)
