"""Weights that are not finite, in the norm without its 8-bit form."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [45, 512, 3000, 16384, 16385, 20000])
def test_infinite_weights_give_infinities_of_the_elements_sign(dtype, cols):
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, w = torch.randn(3, cols, device="cuda", generator=g).to(dtype), torch.ones(cols, device="cuda")
    x[x == 0] = 1.0
    w[::7], w[3::7], w[5::11] = float("inf"), -float("inf"), float("nan")
    y, _, r = api.rms_norm(x, None, w)
    want = x.double() * r.double()[:, None] * w.double()
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.isinf(), want.isinf())
    assert torch.equal(y[y.isinf()].double(), want[want.isinf()])
