"""What the gradient list refuses about its own memory, the norm's and the workspace's: on the C entry points, without a GPU; every check comes before a launch."""
import ctypes as C

import pytest

from paper_1901_06773_amd import binding as B

L = B.lib()


def make(src, counts, at, dst=None):
    k = len(src)
    counts = (C.c_size_t * k)(*counts)
    return L.acc_op_tensor_list((C.c_void_p * k)(*src), (C.c_void_p * k)(*dst) if dst else None, counts, (C.c_int32 * k)(*[B.F32] * k), k, at,
                                L.acc_op_tensor_list_bytes(counts, k), None)


@pytest.mark.parametrize("bad", [
    dict(src=[0x10000], counts=[64], at=0x10000),                                 # the list over a tensor that is scaled in place
    dict(src=[0x10000], counts=[64], at=0x10000 + 240),                           # over its end
    dict(src=[0x10000, 0x20000], counts=[64, 64], at=0x20000 - 64),               # its own end over the second one
    dict(src=[0x10000], counts=[64], dst=[0x30000], at=0x10000),                  # over one that is only read
    dict(src=[0x10000], counts=[64], dst=[0x30000], at=0x30000),                  # over an output
])
def test_the_lists_memory_over_a_tensor(bad):
    assert make(**bad) == B.ACC_EINVAL and "overlap" in L.acc_last_error(None).decode()


NEED = L.acc_op_grad_norm_workspace()


@pytest.mark.parametrize("list_,norm,ws", [(0x100000, 0x100000, 0x200000), (0x100000, 0x100000 + 1008, 0x200000), (0x100000, 0x300000, 0x100000),
                                           (0x100000, 0x300000, 0x100000 - NEED + 16), (0x100000, 0x200000, 0x200000),
                                           (0x100000, 0x200000 + NEED - 16, 0x200000)])
def test_list_norm_and_workspace_over_one_another(list_, norm, ws):
    assert L.acc_op_grad_norm(list_, 1024, norm, ws, NEED, None) == B.ACC_EINVAL
    assert "acc_op_grad_norm" in L.acc_last_error(None).decode() and "overlap" in L.acc_last_error(None).decode()
    assert L.acc_op_grad_clip(list_, 1024, 1.0, norm, ws, NEED, None) == B.ACC_EINVAL
    assert "acc_op_grad_clip" in L.acc_last_error(None).decode() and "overlap" in L.acc_last_error(None).decode()
