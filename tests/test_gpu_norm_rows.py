"""The norm and its gradient with as many rows as there can be."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu


def test_the_most_rows():
    """All rows are zeros but the first and the last two."""
    build.build()
    rows = (1 << 31) - 1
    x = torch.zeros(rows, 1, device="cuda", dtype=torch.bfloat16)
    x[0], x[-2], x[-1] = 3.0, -2.0, 0.5
    w = torch.full((1,), 2.0, device="cuda")
    y, s, r = api.rms_norm(x, None, w, eps=1e-6)
    at = [0, rows - 2, rows - 1]
    assert s is x and y[at, 0].tolist() == [2.0, -2.0, 2.0] and int(y.count_nonzero()) == 3
    dy = y
    dy[1] = 5.0                                           # a row of zeros gets r w dy
    dx, dw = api.rms_norm_grad(dy, None, x, w, r, out=dy)
    assert abs(float(dw[0]) - (2.0 + 2.0 + 2.0)) < 1e-4   # s r = 1, -1, 1
    assert abs(float(dx[1, 0]) / 1e4 - 1) <= 2.0 ** -8 and float(dx[at].abs().max()) < 1e-4
    assert int(dx[2:-2].count_nonzero()) == 0
