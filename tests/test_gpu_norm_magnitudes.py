"""The norm's gradient where r^2 leaves fp32 and r does not, against 64 bits."""
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


def gradient_agrees(dx, dw, dy, ds, s, w, rstd):
    """From the rstd that the kernel is given.  z = s r, the row's sum (80 + cols / 1024 additions one after another),
    its factor and the last products are below 90 + cols / 1024 roundings of each term."""
    e = (90 + s.shape[-1] / 1024) * U
    S, G, r = s.double(), dy.double() * w.double(), rstd.double()[..., None]
    z = S * r
    want = r * (G - z * (G * z).mean(-1, keepdim=True))
    size = r * (G.abs() + z.abs() * (G * z).abs().mean(-1, keepdim=True))
    if ds is not None:
        want, size = want + ds.double(), size + ds.double().abs()
    ok = ((dx.double() - want).abs() <= e * size + R.ROUND[dx.dtype] * want.abs() + 1e-37).all()
    terms = (dy.double() * z)
    ok &= ((dw.double() - terms.sum(0)).abs() <= (len(s) + 3) * U * terms.abs().sum(0) + R.ROUND[dw.dtype] * terms.sum(0).abs()).all()
    return bool(ok)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cols", [40, 45, 512, 1000, 2048, 8000, 16384, 17000])
@pytest.mark.parametrize("size,eps", [(0.0, 1e-40), (3e-20, 0.0), (3e-20, 1e-40), (1e18, 1e-6), (1.0, 1e-6)])
def test_gradients(dtype, cols, size, eps):
    """Zero rows (padding) with r = 1e20, rows whose r is 3e19, and rows of 1e18, whose r^3 and even r^2 times dy
    are below fp32's normal numbers."""
    if size == 1e18 and cols > 300:
        size = 1e17                                   # the sum of squares stays in fp32
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, dy, ds = (torch.randn(6, cols, device="cuda", generator=g) for _ in range(3))
    x = (x * size).to(dtype)
    dy = (dy * (1.0 if size < 1 else 1e-3)).to(dtype)
    ds = (ds * (1e19 if size < 1e-3 else 1e-20 if size > 1e3 else 1.0)).to(dtype)
    w = (1 + 0.3 * torch.randn(cols, device="cuda", generator=g)).to(dtype)
    y, s, r = api.rms_norm(x, None, w, eps=eps)
    assert bool(r.isfinite().all())
    for h in (ds, None):
        dx, dw = api.rms_norm_grad(dy, h, s, w, r)
        assert bool(dx.isfinite().all()) and gradient_agrees(dx, dw, dy, h, s, w, r)
