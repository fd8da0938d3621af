"""Attention whose tanh cap is far above the scores, forward and backward,
against the 64-bit implementation: the cap then hardly changes anything, and
neither pass may lose the scores beside it."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build
from test_gpu_scored import check, make

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
CAPS = [64.0, 65.0, 1e3, 1e4, 1e5, 1e6, 1e8]


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 48)])
@pytest.mark.parametrize("L,bias,causal", [(100, "bucket", False), (330, "none", True), (330, "distance", True),
                                           (290, "bucket", True)])
def test_caps_above_the_scores(L, bias, causal, dtype, D, cap):
    check(*make(2, L, 4, 2, D, dtype, seed=3, bias=bias, causal=causal, cap=cap, docs="packed"))


@pytest.mark.parametrize("cap", [100.0, 1e4, 1e6])
@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 64)])
def test_one_row_near_the_cap_among_ordinary_ones(dtype, D, cap):
    """One query's scores come near the cap; those of its neighbours, in the
    same tile, stay ordinary.  Its dout is zero: fp32 holds no probabilities of
    scores that large, the neighbours' bounds are the usual ones."""
    x, how = make(1, 300, 4, 2, D, dtype, seed=7, causal=True, cap=cap)
    i, j, scale = 140, 130, D ** -0.5
    for h in range(4):
        k = x["k"][0, j, h // 2].float()
        x["q"][0, i, h] = (k * (0.8 * cap / (scale * (k * k).sum()))).to(dtype)
    x["dout"][0, i] = 0
    check(x, how)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("D", [64, 96])
def test_scores_beyond_the_cap_in_fp32(D, seed):
    """Scores of several times the cap, where the cap's derivative is small and has to be as exact as the rest."""
    check(*make(6, 112, 4, 2, D, F32, seed=100 + seed, bias="distance", causal=True, cap=2.0, scale=1.0, docs="mixed"))
