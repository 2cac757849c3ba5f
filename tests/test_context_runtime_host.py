"""What the runtime around the decode step refuses or takes as given, without a GPU."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2606_30389_amd import _lib as L
from paper_2606_30389_amd import runtime as R


@pytest.mark.parametrize("over", [dict(max_kv=4096), dict(max_kv=4999), dict(max_q=4), dict(max_q=0), dict(total_q=7), dict(total_q=0)])
def test_bounds_of_a_batch_hold_its_lengths(over):
    """Bounds below the lengths would have the device cut them: other positions, rows left out."""
    table = torch.zeros(2, 400, dtype=torch.int32)
    with pytest.raises(ValueError):
        R.Batch("cpu", [5, 3], [5000, 3000], table, **over)
    b = R.Batch("cpu", [5, 3], [5000, 3000], table, max_kv=5000, max_q=5, total_q=8)
    assert (b.native.max_kv, b.native.max_q, b.native.total_q) == (5000, 5, 8)
