"""What the top logits and the distillation loss refuse, on the C entry points, without a GPU: every check comes before a launch."""
import pytest

from paper_1901_06773_amd import binding as B

L = B.lib()
BIG = 1 << 40


def at(k):
    return k << 44            # far from one another; nothing reads them


TOP = dict(z=at(1), index=at(2), top=at(3), n=4, classes=10, k=3, ws=at(4), size=BIG, dtype=B.F32)
DIS = dict(z=at(1), index=at(2), top=at(3), labels=at(4), ignore=-1, temperature=2.0, alpha=0.5, rows=at(5), loss=at(6), dz=at(7), n=4, classes=10, k=3, ws=at(8),
           size=BIG, dtype=B.BF16)


def refused(fn, good, **bad):
    rc = fn(*{**good, **bad}.values(), None)
    assert rc == B.ACC_EINVAL, (bad, rc)
    assert fn.__name__ in L.acc_last_error(None).decode()


@pytest.mark.parametrize("bad", [dict(z=None), dict(index=None), dict(top=None), dict(n=0), dict(classes=0), dict(k=0), dict(k=11), dict(n=-1),
                                 dict(classes=(1 << 20) + 1), dict(n=(1 << 20) + 1), dict(classes=5000, k=1025), dict(dtype=2), dict(z=at(1) + 4), dict(top=at(3) + 8),
                                 dict(n=300, classes=1 << 20, k=20, size=1024), dict(n=300, classes=1 << 20, ws=None, size=0), dict(n=1 << 20, classes=1 << 20),
                                 dict(index=at(1)), dict(top=at(2) + 16), dict(ws=at(2), size=64), dict(top=at(1) + 96)])
def test_top_logits(bad):
    refused(L.acc_op_top_logits, TOP, **bad)


@pytest.mark.parametrize("bad", [dict(z=None), dict(index=None), dict(top=None), dict(ws=None), dict(rows=None, loss=None, dz=None), dict(n=0), dict(classes=0),
                                 dict(k=0), dict(k=1025), dict(n=(1 << 20) + 1), dict(classes=(1 << 20) + 1), dict(size=4), dict(dtype=-1), dict(temperature=0.0),
                                 dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(alpha=0.0), dict(alpha=-0.5),
                                 dict(alpha=1.5), dict(alpha=float("nan")), dict(labels=None), dict(z=at(1) + 2), dict(labels=at(4) + 4), dict(dz=at(7) + 8),
                                 dict(n=1 << 20, classes=1 << 20), dict(dz=at(1) + 16), dict(rows=at(4)), dict(loss=at(5)), dict(ws=at(7), size=4096), dict(dz=at(3))])
def test_distillation(bad):
    refused(L.acc_op_distill, DIS, **bad)


def test_refused_sizes_have_no_workspace():
    assert L.acc_op_distill_workspace(4, 10, 3, B.F32) > 0
    for n, classes, k, dtype in ((0, 10, 3, 0), (4, 0, 3, 0), (4, 10, 0, 0), (4, 10, 1025, 0), (4, 10, 3, 2), (4, (1 << 20) + 1, 3, 0)):
        assert L.acc_op_distill_workspace(n, classes, k, dtype) == 0
        assert L.acc_op_top_logits_workspace(n, classes, k, dtype) == 0
    # rows that fit the registers of one workgroup need none, longer ones a list for each segment
    assert L.acc_op_top_logits_workspace(64, 65000, 64, B.F32) == 0
    assert L.acc_op_top_logits_workspace(64, 200000, 64, B.F32) >= 2 * 64 * 4 * 64 * 4


@pytest.mark.parametrize("temperature", [9e-19, 1.1e18, 1e-45, 3e38])
def test_a_temperature_whose_square_is_no_fp32_number_is_refused(temperature):
    refused(L.acc_op_distill, DIS, temperature=temperature)
