"""Workspaces of the norm's gradient at the ends of its range, without a GPU."""
import pytest

from paper_2504_13850_gb300 import api, build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()


@pytest.mark.parametrize("cols", [1, 8, 512, 1024, 1025, 1 << 20])
def test_the_last_rows_below_2_to_31_have_a_workspace(cols):
    most = api.lib().fo_rms_norm_workspace(1 << 20, cols)
    assert most > 0
    for rows in ((1 << 31) - 9, (1 << 31) - 8, (1 << 31) - 7, (1 << 31) - 1):
        assert api.lib().fo_rms_norm_workspace(rows, cols) == most
    assert api.lib().fo_rms_norm_workspace(1 << 31, cols) == -1
