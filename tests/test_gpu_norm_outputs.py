"""The tensors that a norm without a residual writes and returns."""
import pytest
import torch

import scored_reference as R
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [45, 512, 3000, 20000])
def test_sum_out_without_a_residual_holds_x(dtype, cols):
    x, w = torch.randn(5, cols, device="cuda").to(dtype), torch.randn(cols, device="cuda")
    before, want = x.clone(), api.rms_norm(x, None, w)
    # a row whose accesses are not 16 bytes wide is summed in another order: r of either is off by the half of its
    # sum's 80 + cols / 1024 roundings and three more (mean, eps, root), y by two products and its rounding beside
    e = ((80 + cols / 1024) / 2 + 3) * 2.0 ** -24
    f = e + 2 * 2.0 ** -24 + R.ROUND[dtype]
    for given in (torch.zeros_like(x), torch.zeros(5, cols + 3, device="cuda", dtype=dtype)[:, 1:-2], x):
        y, s, r = api.rms_norm(x, None, w, sum_out=given)
        assert s is given and torch.equal(s, before)
        for got, first, off in ((y, want[0], f), (r, want[2], e)):
            assert bool(((got - first).double().abs() <= 2.01 * off * first.double().abs()).all())
    with pytest.raises(ValueError):
        api.rms_norm(x, None, w, sum_out=torch.zeros(4, cols, device="cuda", dtype=dtype))


@pytest.mark.parametrize("cols", [512, 20000])
def test_y_in_place_of_x(cols):
    """Refused where x would be returned as s, which the gradient reads; s elsewhere, y may lie in x's place."""
    x, w = torch.randn(5, cols, device="cuda"), torch.randn(cols, device="cuda")
    before, want = x.clone(), api.rms_norm(x, None, w)
    with pytest.raises(ValueError, match="sum_out"):
        api.rms_norm(x, None, w, out=x)
    with pytest.raises(ValueError, match="sum_out"):
        api.rms_norm(x, None, w, out=x.view(5, cols))
    assert torch.equal(x, before)
    y, s, r = api.rms_norm(x, None, w, out=x, sum_out=torch.empty_like(x))
    assert y is x and torch.equal(s, before) and torch.equal(y, want[0]) and torch.equal(r, want[2])
    assert api.rms_norm(x[:0], None, w, out=x[:0])[0].shape == (0, cols)
