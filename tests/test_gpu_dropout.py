"""Counter-based dropout on the GPU against the plain implementation: equal
masks, one rounding of the result, strides, in place, gradients."""
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


def expect(x, residual, p, seed, call):
    keep, scale = R.dropout_mask(x.numel(), p, seed, call)
    keep = torch.from_numpy(keep).cuda().view(x.shape)
    y = torch.where(keep, x.double() * scale, 0.0)
    size = y.abs()
    if residual is not None:
        y, size = y + residual.double(), size + residual.double().abs()
    # the result's rounding, and fp32 roundings of the product and the sum
    return y, R.ROUND[x.dtype] * y.abs() + 3 * 2.0 ** -24 * size, keep


def agrees(got, want, bound):
    return bool(((got.double() - want).abs() <= bound + 1e-45).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5), (4, 8), (31, 777), (2, 33, 512), (1000, 64), (1, 100003)])
@pytest.mark.parametrize("with_residual", [False, True])
def test_values(dtype, shape, with_residual):
    g = torch.Generator(device="cuda").manual_seed(len(shape))
    x = torch.randn(shape, device="cuda", generator=g).to(dtype)
    r = torch.randn(shape, device="cuda", generator=g).to(dtype) if with_residual else None
    for p, seed, call in ((0.1, 1, 0), (0.5, 2**63 + 11, 2**40 + 3)):
        y = api.dropout_add(x, r, p, seed, call)
        want, bound, _ = expect(x, r, p, seed, call)
        assert agrees(y, want, bound)


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.999999, 1.0])
def test_limits_of_p(p):
    x, r = torch.randn(100, 24, device="cuda"), torch.randn(100, 24, device="cuda")
    y = api.dropout_add(x, r, p, 3, 4)
    want, bound, _ = expect(x, r, p, 3, 4)
    assert agrees(y, want, bound)
    assert p not in (0.0, 1.0) or torch.equal(y, x + r if p == 0.0 else r)


def test_dropped_infinities_do_not_spread():
    x = torch.full((64, 64), float("nan"), device="cuda", dtype=BF)
    x[::2] = float("inf")
    r = torch.ones_like(x)
    y = api.dropout_add(x, r, 0.5, 5, 6)
    keep = expect(torch.ones_like(x), None, 0.5, 5, 6)[2]
    assert bool((y[~keep] == 1).all()) and not bool(torch.isfinite(y[keep]).any())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols,pad,skip", [(5, 64, 8, 0), (33, 40, 3, 0), (17, 64, 8, 1), (9, 1, 6, 2)])
def test_row_strides(dtype, rows, cols, pad, skip):
    """The mask goes by the element's place in the matrix, not in memory."""
    big = [torch.randn(rows, cols + pad, device="cuda").to(dtype) for _ in range(3)]
    x, r, out = (t[:, skip:skip + cols] for t in big)
    before = big[2].clone()
    y = api.dropout_add(x, r, 0.25, 7, 8, out=out)
    want, bound, _ = expect(x, r, 0.25, 7, 8)
    assert agrees(y, want, bound)
    before[:, skip:skip + cols] = y
    assert torch.equal(before, big[2])                      # nothing between the rows was written
    one = torch.randn(1, cols, device="cuda").to(dtype)
    y = api.dropout_add(x, one.expand(rows, cols), 0.25, 7, 8)
    assert agrees(y, *expect(x, one.expand(rows, cols), 0.25, 7, 8)[:2])


def test_in_place():
    x, r = (torch.randn(64, 128, device="cuda") for _ in range(2))
    y = api.dropout_add(x, r, 0.1, 9, 1)
    for target in ("x", "r"):
        a, b = x.clone(), r.clone()
        api.dropout_add(a, b, 0.1, 9, 1, out=a if target == "x" else b)
        assert torch.equal(a if target == "x" else b, y)


def test_gradient_is_the_forward_mask():
    """y is linear in x, so differences with any step give the gradient: dx = keep(dy)."""
    x, d, dy = (torch.randn(50, 72, device="cuda") for _ in range(3))
    dx = api.dropout_grad(dy, 0.3, 10, 2)
    want, bound, _ = expect(dy, None, 0.3, 10, 2)
    assert agrees(dx, want, bound)
    y0, y1 = (api.dropout_add(x + t * d, None, 0.3, 10, 2).double() for t in (-0.5, 0.5))
    diff = float(((y1 - y0) * dy.double()).sum())
    got = float((dx.double() * d.double()).sum())
    assert abs(diff - got) <= 1e-6 * float((dx.double() * d.double()).abs().sum()) + 1e-4


def test_masks_differ_by_call_and_seed_and_keep_the_rate():
    x = torch.ones(1 << 20, device="cuda")
    a, b, c = (api.dropout_add(x, None, 0.1, s, k) != 0 for s, k in ((1, 1), (1, 2), (2, 1)))
    for m in (a, b, c):
        # binomial: 5 standard deviations of the kept share
        assert abs(float(m.double().mean()) - (1 - 6554 / 65536)) < 5 * (0.09 / (1 << 20)) ** 0.5
    for m, n in ((a, b), (a, c)):
        assert abs(float((m & n).double().mean()) - (1 - 6554 / 65536) ** 2) < 5 * (0.16 / (1 << 20)) ** 0.5


def test_elements_beyond_32_bits():
    n = (1 << 32) + 40
    x = torch.ones(n, device="cuda", dtype=BF)
    api.dropout_add(x, None, 0.5, 12, 3, out=x)
    first = n // 8 * 8 - 4096
    g = np.arange(first // 8, (n + 7) // 8, dtype=np.uint64)
    M, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    w = R.philox(np.stack([g & M, g >> s, np.full_like(g, 3), np.zeros_like(g)], 1), (12, 0))
    half = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(-1)[: n - first]
    assert torch.equal(x[first:].float().cpu(), torch.from_numpy(np.where(half >= 32768, 2.0, 0.0)).float())


def test_zero_sizes_and_refusals():
    assert api.dropout_add(torch.empty(0, 4, device="cuda"), None, 0.5, 1, 1).shape == (0, 4)
    assert api.dropout_add(torch.empty(4, 0, device="cuda"), None, 0.5, 1, 1).shape == (4, 0)
    x = torch.ones(4, 8, device="cuda")
    with pytest.raises(api.FedOptimaError, match="p must be"):
        api.dropout_add(x, None, 1.5, 1, 1)
    with pytest.raises(api.FedOptimaError, match="p must be"):
        api.dropout_add(x, None, float("nan"), 1, 1)
    with pytest.raises(api.FedOptimaError, match="stride"):
        api.dropout_add(x, None, 0.5, 1, 1, out=torch.ones(1, 8, device="cuda").expand(4, 8))
    with pytest.raises(ValueError):
        api.dropout_add(x, x[:2], 0.5, 1, 1)
    with pytest.raises(ValueError):
        api.dropout_add(x.half(), None, 0.5, 1, 1)
    with pytest.raises(ValueError):
        api.dropout_add(x.cpu(), None, 0.5, 1, 1)
    with pytest.raises(ValueError):
        api.dropout_add(x.t(), None, 0.5, 1, 1)
