"""What the gated layer refuses, on the C entry points, without a GPU: every check comes before a launch."""
import pytest

from paper_1901_06773_amd import binding as B

L = B.lib()
BIG = 1 << 50


def at(k):
    return k << 52            # far from one another; nothing reads them


FWD = dict(x=at(1), w=at(2), bias=None, h=at(3), ab=None, rows=40, d=16, f=8, act=2, ws=at(4), size=BIG, dtype=B.BF16)
BWD = dict(x=at(1), w=at(2), bias=at(3), ab=None, dh=at(4), dx=at(5), dw=at(6), db=at(7), rows=40, d=16, f=8, act=2, ws=at(8), size=BIG, dtype=B.F32)


def refused(fn, good, **bad):
    rc = fn(*{**good, **bad}.values(), None)
    assert rc == B.ACC_EINVAL, (bad, rc)
    assert fn.__name__ in L.acc_last_error(None).decode()


COMMON = [dict(x=None), dict(w=None), dict(rows=0), dict(d=0), dict(f=0), dict(rows=-3), dict(rows=(1 << 24) + 1), dict(d=(1 << 16) + 1), dict(f=(1 << 16) + 1),
          dict(d=1 << 15, f=1 << 15), dict(d=1 << 16, f=1 << 16), dict(rows=1 << 24, d=1 << 13), dict(act=3), dict(act=-1), dict(dtype=2), dict(x=at(1) + 8), dict(w=at(2) + 2)]


@pytest.mark.parametrize("bad", COMMON + [dict(h=None), dict(h=at(3) + 4), dict(ab=at(5) + 8), dict(rows=3000, d=513, f=33, size=16), dict(d=17, ws=None),
                                          dict(h=at(1)), dict(h=at(2) + 64), dict(ab=at(3) + 512), dict(ab=at(4), size=4096), dict(bias=at(3) + 16)])
def test_forward(bad):
    refused(L.acc_op_glu_fwd, FWD, **bad)


@pytest.mark.parametrize("bad", COMMON + [dict(dh=None), dict(ws=None), dict(size=64), dict(dx=None, dw=None, db=None), dict(dw=at(6) + 4), dict(dx=at(1)), dict(dx=at(4) + 32),
                                          dict(dw=at(2)), dict(db=at(3)), dict(ab=at(5)), dict(db=at(6) + 16), dict(ws=at(5), size=1 << 30)])
def test_backward(bad):
    refused(L.acc_op_glu_bwd, BWD, **bad)


def test_workspaces():
    assert L.acc_op_glu_workspace(4, 512, 2048, 0, B.BF16) == 0 and L.acc_op_glu_workspace(4, 512, 2048, 1, B.BF16) > 0
    for rows, d, f, dtype in ((0, 4, 4, 0), (4, 0, 4, 0), (4, 4, 0, 0), (4, 4, 4, 5), (4, 1 << 16, 1 << 16, 1)):
        assert L.acc_op_glu_workspace(rows, d, f, 1, dtype) == 0
    # widths of no whole eights are copied, whole ones are not
    assert L.acc_op_glu_workspace(100000, 1024, 4096, 0, B.BF16) == 0 and L.acc_op_glu_workspace(100000, 1023, 4096, 0, B.BF16) >= 100000 * 1024 * 2
