"""Orthogonalised updates of fp32 matrices in which one row (or column) is far smaller
than the others, row by row against 64 bits."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()
    yield
    api.orthogonalize_error()


def weak_row_bound(X, row):
    """(X after five steps, bound of one row's error in its 2-norm) from U / |U| with rows <= columns, in 64 bits.

    What is relative: X's storage 2^-23, and of A, C and C X fewer than 14 * 2^-23 each of their row (truncated
    products of 64 terms, their sum in fp32, storage); C X stays below a X in a weak row: 16 * 2^-23 per step.
    What is absolute: an element of X is off by 2^-46 at least, one of A and of C by 2^-44, of random sign, so that
    a row of them times X is off by sqrt(m) 2^-44 |X|_2, A's times |b| + |c| |A| < 8.  An error of a weak row grows
    like the row, at most by a = 3.4445 a step."""
    a, b, c = api.QUINTIC
    m, n = X.shape
    e = n ** 0.5 * 2.0 ** -46
    for _ in range(5):
        A = X @ X.t()
        S = float(torch.linalg.eigvalsh(A)[-1].clamp(min=0).sqrt())
        e = a * (e + 16 * 2.0 ** -23 * float(X[row].norm())) + n ** 0.5 * 2.0 ** -46 + 9 * m ** 0.5 * 2.0 ** -44 * S
        X = a * X + (b * A + c * A @ A) @ X
    return X, e


@pytest.mark.parametrize("rows,cols", [(512, 2048), (100, 300), (300, 200), (200, 96), (30, 70), (260, 260)])
@pytest.mark.parametrize("power", [0, 2, 3, 4, 5, 6])
def test_a_weak_row_keeps_its_bits(rows, cols, power):
    g = torch.Generator(device="cuda").manual_seed(power)
    u = torch.randn(rows, cols, device="cuda", generator=g)
    weak = u if rows <= cols else u.t()                   # a row of what is iterated on
    weak[min(rows, cols) // 3] *= 10.0 ** -power
    x = weak.double()
    want, e = weak_row_bound(x / (x.norm() + 1e-7), min(rows, cols) // 3)
    got = api.orthogonalize(u)
    got = got if rows <= cols else got.t()
    row = min(rows, cols) // 3
    assert float((got[row].double() - want[row]).norm()) <= e
