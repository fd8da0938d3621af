"""Orthogonalised updates on the GPU at the accuracy that their roundings give, block
by block, against an emulation of these roundings and 64 bits."""
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


def make(rows, cols, dtype, seed=0, spread=True):
    return E.make(rows, cols, dtype, seed, spread, "cuda")


# in shared memory (one CTA and several, either side the longer); tiles of pairs; shared sums; wide tiles in two rounds
SHAPES = [(40, 65), (63, 65), (64, 64), (96, 200), (200, 96), (128, 128), (128, 2048), (1000, 77), (70, 700),
          (129, 127), (130, 384), (150, 300), (320, 200), (512, 513), (100, 2049), (1300, 128), (140, 4096), (512, 2048), (2048, 512),
          (700, 1100), (1536, 512), (1000, 1000)]


@pytest.mark.parametrize("spread", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_values(dtype, rows, cols, spread):
    u = make(rows, cols, dtype, spread=spread)
    assert E.Held(u, dtype, dtype == F32).why_not(api.orthogonalize(u)) is None


@pytest.mark.parametrize("rows,cols,dtype", [(2400, 2400, BF), (2600, 2500, BF), (2900, 2900, BF), (1900, 2100, F32)])
def test_more_tiles_than_pairs(rows, cols, dtype):
    u = make(rows, cols, dtype)
    assert E.Held(u, dtype, dtype == F32).why_not(api.orthogonalize(u)) is None


@pytest.mark.parametrize("dtype", [F32, BF])
def test_lists(dtype):
    us = [make(r, c, dtype, seed=k) for k, (r, c) in enumerate([(1500, 1700), (700, 2400), (1300, 1000), (40, 90), (200, 96), (512, 512)])]
    for u, x in zip(us, api.orthogonalize(us)):
        assert E.Held(u, dtype, dtype == F32).why_not(x) is None, tuple(u.shape)


@pytest.mark.parametrize("steps,coefficients", [(1, E.QUINTIC), (2, E.QUINTIC), (8, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0))])
@pytest.mark.parametrize("rows,cols", [(90, 200), (300, 260)])
def test_other_polynomials(rows, cols, steps, coefficients):
    u = make(rows, cols, F32)
    how = dict(steps=steps, coefficients=coefficients, eps=1e-3)
    assert E.Held(u, F32, True, **how).why_not(api.orthogonalize(u, **how)) is None


@pytest.mark.parametrize("dtype", [F32, BF])
def test_updates_of_parameters(dtype):
    """Of a step without decay on parameters of zeros, with the momentum of an earlier step."""
    shapes = [(150, 300), (96, 200), (200, 96), (700, 512)]
    params = [torch.zeros(s, device="cuda") for s in shapes]
    grads = [make(*s, dtype, seed=k) for k, s in enumerate(shapes)]
    momenta = [make(*s, F32, seed=50 + k) for k, s in enumerate(shapes)]
    api.muon_step(params, grads, momenta, 1.0, momentum=0.5, scales=[1.0] * len(shapes))
    for p, g, m in zip(params, grads, momenta):
        assert E.Held((g.float() + 0.5 * m), F32, True).why_not(-p) is None
