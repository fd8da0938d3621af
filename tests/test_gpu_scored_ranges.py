"""Attention at the ends of what its arguments may be: scales and caps near the
limits of fp32."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build
from test_gpu_scored import check, make

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 32)])
@pytest.mark.parametrize("bias", ["none", "distance", "bucket"])
@pytest.mark.parametrize("scale,cap", [(1e-39, 0.0), (1e-36, 0.0), (1e-20, 0.0), (1e25, 0.0), (0.1, 1e-39), (0.1, 1e-30),
                                       (0.1, 1e30), (0.1, 3e38), (1e-39, 1e-39), (1e-39, 3e38)])
def test_scales_and_caps_near_the_limits(scale, cap, bias, dtype, D):
    """Scores stay ordinary (queries shrink as the scale grows) or vanish."""
    x, how = make(2, 200, 4, 2, D, dtype, seed=13, bias=bias, causal=True, cap=cap, scale=scale, docs="padded")
    if scale > 1:
        x["q"] = (x["q"].float() / (scale * D ** 0.5)).to(dtype)
    x["q"][:, 5] = 0
    check(x, how)
