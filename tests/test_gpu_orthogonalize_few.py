"""Orthogonalised updates of bf16 matrices with a side of up to 16 elements: off by
their own rounding and no more."""
import pytest
import torch

import orthogonalize_emulation as E
from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()
    yield
    api.orthogonalize_error()


@pytest.mark.parametrize("spread", [True, False])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 3), (8, 8), (15, 15), (16, 16), (15, 9), (9, 37), (16, 200), (300, 12), (16, 3000), (5000, 7)])
def test_the_results_rounding_is_what_is_lost(rows, cols, spread):
    """Before it an element is off by d: of the norm, 16 * 2^-23 per step and a slope of 4 at most.  An element that is
    rounded to the other side for it lay within d of the middle: at most 2 d are added to its rounding's error."""
    for seed in range(8):
        u = E.make(rows, cols, torch.bfloat16, seed, spread, "cuda")
        want = E.exact(u)
        own = float((want.bfloat16().double() - want).norm())
        off = float((api.orthogonalize(u).double() - want).norm())
        assert off <= own + 2 * (5 * 4 * 16 * 2.0 ** -23) * float(want.norm()), (seed, off / own)
