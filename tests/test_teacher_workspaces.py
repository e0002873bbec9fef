"""Sizes at the limits that the header states, and what the workspaces hold, on the C entry points, without a GPU."""
import pytest

from paper_1901_06773_amd import binding as B

L = B.lib()


@pytest.mark.parametrize("dtype,each", [(B.F32, 16448), (B.BF16, 32896)])
def test_distillation_has_fewer_than_2_to_the_22_workgroups(dtype, each):
    classes = 1 << 20
    parts = -(-classes // each)
    most = ((1 << 22) - 1) // parts
    assert L.acc_op_distill_workspace(most, classes, 4, dtype) > 0
    assert L.acc_op_distill_workspace(most + 1, classes, 4, dtype) == 0
    assert L.acc_op_distill_workspace(1 << 20, 65000, 4, dtype) > 0      # (a workgroup per row)
