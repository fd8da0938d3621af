"""Orthogonalised updates at the ends of their range: sides of 32768 and 2^20, offsets
beyond 32 bits, and two calls at the same time."""
import pytest
import torch

import orthogonalize_emulation as E
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()
    yield
    api.orthogonalize_error()


def polynomial(x, steps=5):
    """Of singular values."""
    a, b, c = api.QUINTIC
    for _ in range(steps):
        x = x * (a + b * x ** 2 + c * x ** 4)
    return x


@pytest.mark.parametrize("rows,cols,dtype", [(32768, 32768, BF), (16000, 32768, F32), (300, 1 << 20, F32), (1 << 20, 200, BF), (1 << 20, 40, F32),
                                             (1, 1 << 20, F32)])
def test_longest_sides(rows, cols, dtype):
    """One nonzero per row of the shorter side, at random places of the longer one: each has the polynomial of its
    own value, every other element stays zero.  Of pairs fewer than 16 * 2^-23 are lost in a step, of a single
    operand's polynomial 8 * 2^-12, and both pass on with a slope of at most 4 of their size."""
    n = min(rows, cols)
    g = torch.Generator(device="cuda").manual_seed(1)
    long = torch.randperm(max(rows, cols), device="cuda", generator=g)[:n]
    i, j = (torch.arange(n, device="cuda"), long) if rows <= cols else (long, torch.arange(n, device="cuda"))
    u = torch.zeros(rows, cols, device="cuda", dtype=dtype)
    u[i, j] = torch.linspace(0.5, 1.5, n, device="cuda").to(dtype)
    got = api.orthogonalize(u)
    x = u[i, j].double()
    x = polynomial(x / (x.norm() + 1e-7))
    off = 5 * 4 * (16 * 2.0 ** -23 if dtype == F32 else 8 * 2.0 ** -12) + (2.0 ** -24 if dtype == F32 else 2.0 ** -8)
    assert bool(((got[i, j].double() - x).abs() <= off * x.abs()).all())
    got[i, j] = 0
    assert not bool(got.any())


@pytest.mark.parametrize("rows,cols", [(300, 200), (200, 300), (130, 100)])
def test_offsets_beyond_32_bits(rows, cols):
    """Rows 2^24 elements apart, in every tensor that has rows."""
    stride = (1 << 24) + 8

    def far(t):
        big = torch.empty((rows - 1) * stride + cols, device="cuda", dtype=t.dtype).as_strided((rows, cols), (stride, 1))
        return big.copy_(t)

    u = E.make(rows, cols, BF, device="cuda")
    want = api.orthogonalize(u)
    out = far(torch.zeros_like(u))
    assert torch.equal(api.orthogonalize(far(u), out=out), want)
    p, m = torch.randn(rows, cols, device="cuda"), torch.randn(rows, cols, device="cuda")
    P, M = far(p), far(m)
    for params, momenta, grads in (([p], [m], [u]), ([P], [M], [far(u)])):
        api.muon_step(params, grads, momenta, 0.1, momentum=0.5, weight_decay=0.3)
    assert torch.equal(P, p) and torch.equal(M, m)


def test_two_calls_at_once():
    """Lists in shared memory, of tiles and of both types on two streams, over and over."""
    lists = [[E.make(r, c, t, seed=k, device="cuda") for k, (r, c) in enumerate(shapes)]
             for t, shapes in ((F32, [(200, 96), (512, 2048), (700, 700)]), (BF, [(100, 60), (1500, 1000), (128, 2048)]))]
    want = [api.orthogonalize(us) for us in lists]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in lists], [[], []]
    for _ in range(20):
        for us, s, to in zip(lists, streams, got):
            with torch.cuda.stream(s):
                to.append(api.orthogonalize(us))
    torch.cuda.synchronize()
    for w, to in zip(want, got):
        assert all(torch.equal(x, y) for xs in to for x, y in zip(xs, w))
