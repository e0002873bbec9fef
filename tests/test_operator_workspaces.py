"""Workspace sizes and refusals agree, on the C entry points and without a GPU: nothing here reaches a device."""
import pytest

from paper_1901_06773_amd import binding as B

L = B.lib()


def at(k):
    return k << 44            # far from one another; nothing reads them


def gn_forward(n, hw, c, groups, size, dtype):
    return L.acc_op_gn_fwd(at(1), at(2), at(3), None, at(4), at(5), at(6), n, hw, c, groups, 0, 1e-5, at(7), size, dtype, None)


def gn_backward(n, hw, c, groups, size, dtype):
    return L.acc_op_gn_bwd(at(1), at(2), None, None, at(3), at(4), at(5), at(6), at(7), at(8), at(9), None, n, hw, c, groups, 0, at(10), size, dtype, None)


# sizes that one storage type alone would take: a bf16 row of 516 channels is read value by value, in four times the workgroups
@pytest.mark.parametrize("n,hw,c,groups", [(4194304, 1, 516, 4), (4194304, 1, 516, 2), (4194304, 1, 900, 4)])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_group_norm_of_sizes_without_a_workspace_is_refused(n, hw, c, groups, dtype):
    assert L.acc_op_gn_workspace(n, hw, c, groups) == 0
    for size in (16, 1 << 40):
        for call in (gn_forward, gn_backward):
            assert call(n, hw, c, groups, size, dtype) == B.ACC_EINVAL, (call.__name__, size)


@pytest.mark.parametrize("n,hw,c,groups", [(4000000, 1, 516, 4), (1, 1, 1, 1), (3, 49, 30, 3), (64, 3136, 256, 32)])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_group_norm_with_a_smaller_workspace_is_refused(n, hw, c, groups, dtype):
    size = L.acc_op_gn_workspace(n, hw, c, groups)
    assert size > 0
    for call in (gn_forward, gn_backward):
        assert call(n, hw, c, groups, size - 256, dtype) == B.ACC_EINVAL


def ce_bytes(n, d, classes):
    return L.acc_op_linear_ce_workspace(n, d, classes, 1, B.BF16)


@pytest.mark.parametrize("n,d,classes,kept", [(1000, 1024, 1000, False), (64, 1024, 300, False), (41, 2048, 1000, False), (200, 1024, 3000, False),
                                              (4096, 512, 16384, False), (65536, 1024, 1000, False), (131072, 512, 100, False), (777, 512, 50001, True), (6, 216, 49305, True), (16, 640, 100000, True),
                                              (4096, 2048, 16384, True), (777, 1160, 50001, True)])
def test_which_logits_the_linear_cross_entropy_keeps(n, d, classes, kept):
    """Kept logits are the part of the workspace that a loss alone has no use for, beside dz as two or three bf16 values and sums."""
    pitch = -(-classes // 64) * 64
    parts = 3 if n < 4096 else 2
    logits, dz = n * pitch * 4, parts * n * pitch * 2
    # sums of dx and dw in up to 2^25 and 2^24 values, and of db
    least = dz + n * d * 4
    assert ce_bytes(n, d, classes) >= least + (logits if kept else 0)
    if not kept:
        assert ce_bytes(n, d, classes) - ce_bytes(n, d - 16, classes) < logits


def documented(n, d, classes, gradients, dtype):
    """The bound that include/accudnn.h states."""
    width, MiB, GiB = -(-d // 8) * 8, 1 << 20, 1 << 30
    fp32 = dtype == B.F32 or d < 16 or n * width * 2 > 0xFFFFFF00
    total = 16 * n + 65536 + 8 * n * (classes // (32 if fp32 else 64) + 1)
    values = max(1 << 26, 256 * n)
    if gradients:
        total += 10 * values + 4 * n * d + 192 * MiB + 4 * min(n * (classes + 256), values) // 16 + 128 * MiB + 4 * classes
    elif fp32:
        total += 4 * (1 << 24)
    if dtype == B.BF16 and fp32:
        total += 4 * n * d + max(GiB, 4 * 128 * d)
    elif dtype == B.BF16 and d % 8:
        total += 2 * n * width + max(GiB, 2 * 256 * width)
    return total


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("gradients", [0, 1])
def test_the_linear_cross_entropys_workspace_keeps_its_bound(gradients, dtype):
    rows = (1, 2, 41, 512, 777, 4095, 4096, 8192, 65536, 1 << 18, 1 << 20)
    for n in rows:
        for d in (1, 8, 15, 16, 60, 64, 1024, 1160, 4096, 4100, 65536):
            for classes in (1, 2, 100, 1000, 4097, 50001, 65536, 1 << 20, 1 << 24):
                size = L.acc_op_linear_ce_workspace(n, d, classes, gradients, dtype)
                assert 0 < size <= documented(n, d, classes, gradients, dtype), (n, d, classes, size / 2 ** 20)
