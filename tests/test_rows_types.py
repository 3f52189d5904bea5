"""Types of rows that the Python calls take and refuse."""
import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import device
from tests.test_cache_args import _refuses


@pytest.mark.parametrize("x", [torch.zeros((4, 64), dtype=torch.float64), torch.zeros((4, 64), dtype=torch.int32), torch.zeros(64), torch.zeros((2, 2, 2, 2)), None, [1.0]])
def test_a_workspace_for_what_is_no_row(x):
    assert "known type" in _refuses(B.AMAP_E_INVALID, device.norm_grad_workspace, x)


def test_a_workspace_for_rows_of_8_bits():
    _refuses(B.AMAP_E_INVALID, device.norm_grad_workspace, torch.zeros((4, 64), dtype=torch.float8_e4m3fn))
