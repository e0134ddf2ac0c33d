"""The measurement hooks over the layers' calls: how many kernels a call launches, and one tagged pair of events for each."""
import os
import re

import pytest
import torch

from paper_1704_05021_b200 import binding as B
from paper_1704_05021_b200 import layers as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16 = torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("rows, width, dx, sums, launches", [(4, 9000, True, True, 3), (4, 9000, True, False, 1), (4, 9000, False, True, 2), (400, 9000, False, True, 2),
                                                            (0, 9000, True, True, 1), (4, 64, True, True, 1), (40000, 64, False, True, 2), (40000, 64, True, False, 1)])
def test_launches_of_the_norms_backward_pass_are_counted(cuda_device, rows, width, dx, sums, launches):
    """Rows too long to hold: the sums of columns, dx, and the join of the sums are a launch each, where they are wanted."""
    norm = L.LayerNormSession(width, max(rows, 1), dtype=BF16, device=cuda_device)
    x = torch.ones(rows, width, dtype=BF16, device=cuda_device)
    stat = torch.ones(rows, device=cuda_device)
    dw = torch.empty(width, device=cuda_device) if sums else None
    before = B.gd_launch_count()
    norm.backward(x, x, None, stat, stat, dx=torch.empty_like(x) if dx else None, dweight=dw)
    assert B.gd_launch_count() - before == launches
