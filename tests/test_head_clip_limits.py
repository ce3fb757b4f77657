"""Limits that a clipping handle refuses, without a GPU."""
import pytest
import torch

from paper_2407_11698_gb300 import binding as nb


class _Norm:
    """As much of a tensor as a call looks at before it goes to the library."""
    dtype, is_cuda = torch.float32, True

    def numel(self):
        return 1

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("limit", [0.0, -1.0, float("nan"), 1e-46, 7e-46])
def test_limits_that_are_not_above_zero_in_fp32(limit):
    op = object.__new__(nb.GradClip)
    op.h = None
    with pytest.raises(ValueError):
        op.run(_Norm(), limit, stream=0)
