"""What group norm, linear cross-entropy and the gradient list refuse, on the C entry points, without a GPU: every check comes before a
launch, so nothing here reaches a device."""
import ctypes as C

import pytest

from paper_1901_06773_amd import binding as B

L = B.lib()
P, ODD = 4096, 4100           # an aligned address and one that is not; nothing reads them
BIG = 1 << 40


def text():
    return L.acc_last_error(None).decode()


def at(k):
    return k << 44            # far from one another


GN = dict(x=at(1), gamma=at(2), beta=at(3), res=None, y=at(4), mean=at(5), istd=at(6), n=2, hw=9, c=12, groups=3, act=1, eps=1e-5, ws=at(7), size=BIG, dtype=B.F32)
GNB = dict(x=at(1), dy=at(2), y=at(3), res=None, gamma=at(4), beta=at(5), mean=at(6), istd=at(7), dx=at(8), dgamma=at(9), dbeta=at(10), dres=None, n=2,
           hw=9, c=12, groups=3, act=1, ws=at(11), size=BIG, dtype=B.F32)
CE = dict(x=at(1), w=at(2), bias=None, labels=at(3), ignore=-1, rows=at(4), loss=at(5), dx=at(6), dw=at(7), db=at(8), n=4, d=8, classes=5, ws=at(9), size=BIG, dtype=B.BF16)


def refused(fn, good, **bad):
    rc = fn(*{**good, **bad}.values(), None)
    assert rc == B.ACC_EINVAL, (bad, rc)
    assert fn.__name__ in text()


@pytest.mark.parametrize("bad", [dict(x=None), dict(gamma=None), dict(beta=None), dict(y=None), dict(mean=None), dict(istd=None), dict(ws=None),
                                 dict(x=ODD), dict(res=ODD), dict(istd=ODD), dict(ws=ODD), dict(n=0), dict(hw=0), dict(c=0), dict(groups=0), dict(groups=5),
                                 dict(groups=-3), dict(n=-1), dict(act=3), dict(act=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(size=16),
                                 dict(dtype=2), dict(n=1 << 30, groups=12), dict(hw=1 << 30)])
def test_group_norm_forward(bad):
    refused(L.acc_op_gn_fwd, GN, **bad)


@pytest.mark.parametrize("bad", [dict(x=None), dict(dy=None), dict(y=None), dict(gamma=None), dict(beta=None), dict(mean=None), dict(istd=None), dict(dx=None),
                                 dict(dgamma=None), dict(dbeta=None), dict(ws=None), dict(dres=ODD), dict(dy=ODD), dict(groups=7), dict(n=0), dict(hw=-4),
                                 dict(c=0), dict(act=9), dict(size=16), dict(dtype=-1)])
def test_group_norm_backward(bad):
    refused(L.acc_op_gn_bwd, GNB, **bad)


@pytest.mark.parametrize("bad", [dict(x=None), dict(w=None), dict(labels=None), dict(ws=None), dict(rows=None, loss=None, dx=None, dw=None, db=None), dict(n=0),
                                 dict(d=0), dict(classes=0), dict(n=(1 << 20) + 1), dict(d=(1 << 16) + 1), dict(classes=(1 << 24) + 1), dict(size=64),
                                 dict(x=ODD), dict(w=ODD), dict(labels=ODD), dict(dw=ODD), dict(bias=ODD), dict(dtype=7)])
def test_linear_cross_entropy(bad):
    refused(L.acc_op_linear_ce, CE, **bad)


@pytest.mark.parametrize("fn,good,bad", [
    (L.acc_op_gn_fwd, GN, dict(y=at(1) + 16)), (L.acc_op_gn_fwd, GN, dict(mean=at(6))), (L.acc_op_gn_fwd, GN, dict(istd=at(3) + 32)),
    (L.acc_op_gn_fwd, GN, dict(ws=at(1) - 4096)), (L.acc_op_gn_fwd, GN, dict(res=at(4) + 64)),
    (L.acc_op_gn_bwd, GNB, dict(dx=at(3))), (L.acc_op_gn_bwd, GNB, dict(dx=at(2), dres=at(2))), (L.acc_op_gn_bwd, GNB, dict(dres=at(1))),
    (L.acc_op_gn_bwd, GNB, dict(dgamma=at(10))), (L.acc_op_gn_bwd, GNB, dict(dbeta=at(5))), (L.acc_op_gn_bwd, GNB, dict(dx=at(2) + 16)),
    (L.acc_op_gn_bwd, GNB, dict(act=2, y=None, res=at(8))),
    (L.acc_op_linear_ce, CE, dict(dx=at(1))), (L.acc_op_linear_ce, CE, dict(dw=at(2))), (L.acc_op_linear_ce, CE, dict(bias=at(8))),
    (L.acc_op_linear_ce, CE, dict(rows=at(3))), (L.acc_op_linear_ce, CE, dict(db=at(7) + 16)), (L.acc_op_linear_ce, CE, dict(ws=at(2) - 256))])
def test_results_over_other_arguments(fn, good, bad):
    refused(fn, good, **bad)
    assert "overlaps" in text()


def test_workspaces_of_sizes_that_are_refused():
    assert L.acc_op_gn_workspace(0, 1, 1, 1) == L.acc_op_gn_workspace(1, 1, 4, 3) == 0
    assert L.acc_op_linear_ce_workspace(0, 1, 1, 1, 0) == L.acc_op_linear_ce_workspace(1, 1, 1, 1, 2) == 0
    assert L.acc_op_linear_ce_workspace(8, 64, 100, 1, 0) > L.acc_op_linear_ce_workspace(8, 64, 100, 0, 0) > 0
    assert B.op_grad_norm_workspace() > 0


def make_list(src, counts, dst=None, dtypes=None, n=None, size=None, at=P):
    k = len(src)
    counts = (C.c_size_t * k)(*counts)
    need = L.acc_op_tensor_list_bytes(counts, k)
    return L.acc_op_tensor_list((C.c_void_p * k)(*src), (C.c_void_p * k)(*dst) if dst else None, counts, (C.c_int32 * k)(*(dtypes or [B.F32] * k)),
                                k if n is None else n, at, need if size is None else size, None)


@pytest.mark.parametrize("bad", [
    dict(src=[0x10000, None], counts=[4, 4]),                                    # null
    dict(src=[0x10000, 0x20002], counts=[4, 4]),                                 # half an fp32
    dict(src=[0x10000, 0x20001], counts=[4, 4], dtypes=[1, 1]),                  # half a bf16
    dict(src=[0x10000, 0x10000], counts=[4, 4]),                                 # the same tensor twice
    dict(src=[0x10000, 0x1000c], counts=[4, 4]),                                 # the last value of one is the first of the next
    dict(src=[0x10000, 0x20000], counts=[4, 4], dst=[0x30000, 0x30004]),         # outputs overlap
    dict(src=[0x10000, 0x20000], counts=[4, 4], dst=[0x20004, 0x40000]),         # an output over another's input
    dict(src=[0x10000, 0x20000], counts=[4, 4], dst=[0x10004, 0x40000]),         # an output beside its own input
    dict(src=[0x10000], counts=[1 << 20], dst=[0x20000]),                        # the same, far
    dict(src=[0x10000], counts=[4], dtypes=[2]),
    dict(src=[0x10000], counts=[4], n=0),
    dict(src=[0x10000], counts=[4], n=-1),
    dict(src=[0x10000], counts=[4], size=64),
    dict(src=[0x10000], counts=[4], at=None),
    dict(src=[0x10000], counts=[4], at=ODD),
    dict(src=[0x10000], counts=[1 << 45]),
])
def test_tensor_list(bad):
    assert make_list(**bad) == B.ACC_EINVAL
    assert "acc_op_tensor_list" in text()


def test_tensor_list_sizes():
    def size(*counts):
        return L.acc_op_tensor_list_bytes((C.c_size_t * len(counts))(*counts), len(counts))
    assert size(0) == size(0, 0) > 0 and size(1) >= size(0) and size(1 << 45) == 0
    assert size(16384 * 100) < size(16384 * 100 + 16384 * 50) and L.acc_op_tensor_list_bytes(None, 3) == 0


@pytest.mark.parametrize("bad", [dict(at=None), dict(norm=None), dict(ws=None), dict(size=0), dict(room=8), dict(at=ODD), dict(norm=ODD), dict(ws=ODD)])
def test_norm_and_clip(bad):
    a = {**dict(at=P, size=1024, norm=P, ws=P, room=1 << 20), **bad}
    assert L.acc_op_grad_norm(a["at"], a["size"], a["norm"], a["ws"], a["room"], None) == B.ACC_EINVAL and "acc_op_grad_norm" in text()
    assert L.acc_op_grad_clip(a["at"], a["size"], 1.0, a["norm"], a["ws"], a["room"], None) == B.ACC_EINVAL and "acc_op_grad_clip" in text()


@pytest.mark.parametrize("bound", [-1.0, float("nan"), float("-inf")])
def test_clip_bound(bound):
    assert L.acc_op_grad_clip(P, 1024, bound, P, P, 1 << 20, None) == B.ACC_EINVAL
