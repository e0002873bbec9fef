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


@pytest.mark.parametrize("dtype,each", [(B.F32, 16448), (B.BF16, 32896)])
@pytest.mark.parametrize("n,classes,k", [(64, 1000000, 50), (777, 300007, 1024), (4000, 1 << 20, 1)])
def test_what_distillation_keeps_of_cut_rows(n, classes, k, dtype, each):
    def pieces(*sizes):
        return sum((s + 255) // 256 * 256 for s in sizes)
    per = 4 if dtype == B.F32 else 8
    chunks = -(-classes // per) + (1 if classes % per else 0)
    parts = n * -(-chunks // (each // per))
    counts = 256 if n > 65536 else -(-n // 256) if n > 1024 else 0
    # the rows' losses, the counts, three sums of each part and one in 64 bits, the logits of the list and of the label
    assert L.acc_op_distill_workspace(n, classes, k, dtype) == pieces(4 * n, 4 * counts, 3 * 4 * parts, 8 * parts, 4 * n * (k + 1))
