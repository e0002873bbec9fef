"""Gradients and values that are not finite at gates that are closed (ReLU at or below 0, SiLU where the sigmoid is 0 in fp32): db = dh act(a) and da = dh b
act'(a) are 0 times them, which is no number.  What they do not enter keeps its bits.  A gate of minus infinity is closed like any other."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ACT = {"none": 0, "relu": 1, "silu": 2}
CLOSED, OPEN = [0, 2, 4], [1, 3]              # columns
# few rows, fewer columns than a tile of pairs takes, sums in parts, odd widths, each kind of tile, both sides of 4096 rows
SIZES = [(4, 64, 32), (5, 24, 6), (70, 64, 40), (64, 4096, 64), (300, 512, 256), (131, 33, 57), (2009, 256, 136), (4200, 40, 24), (4200, 512, 1024)]


def B():
    from paper_1901_06773_amd import binding
    return binding


def inputs(rows, d, f, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(7)

    def r(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    bias = 0.3 * r(2 * f)
    bias[:f] += 3.0
    bias[torch.tensor(CLOSED)] = -300.0       # the projections have a spread of 1
    return r(rows, d).to(DT[dtype]), (r(2 * f, d) / d ** 0.5).to(DT[dtype]), bias, r(rows, f).to(DT[dtype])


def forward(x, w, bias, act):
    rows, d, f = x.shape[0], x.shape[1], w.shape[0] // 2
    h, ab = torch.empty(rows, f, device="cuda", dtype=x.dtype), torch.empty(rows, 2 * f, device="cuda", dtype=x.dtype)
    ws = torch.empty(max(16, B().op_glu_workspace(rows, d, f, False, B()._dtype_of(x))), dtype=torch.uint8, device="cuda")
    B().op_glu_fwd(x, w, bias, h, ab, ACT[act], ws)
    return h, ab


def backward(x, w, bias, ab, dh, act):
    rows, d, f = x.shape[0], x.shape[1], w.shape[0] // 2
    dx, dw, db = torch.empty_like(x), torch.empty(2 * f, d, device="cuda"), torch.empty(2 * f, device="cuda")
    ws = torch.empty(B().op_glu_workspace(rows, d, f, True, B()._dtype_of(x)), dtype=torch.uint8, device="cuda")
    B().op_glu_bwd(x, w, bias, ab, dh, dx, dw, db, ACT[act], ws)
    return dx, dw, db


def none_at(got, clean, rows, columns):
    """No row of dx in `rows` and no row of dw, no value of db in `columns` is a number; everything else is as it is without what is not finite."""
    for what, v, c, bad in zip(("dx", "dw", "db"), got, clean, (rows, columns, columns)):
        mask = torch.zeros(v.shape[0], dtype=torch.bool, device="cuda")
        mask[torch.tensor(bad, dtype=torch.long)] = True
        assert not torch.isfinite(v[mask]).any(), what
        assert torch.equal(v[~mask], c[~mask]), what


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,f", SIZES)
def test_gradients_that_are_not_finite(rows, d, f, dtype, act, value):
    x, w, bias, dh = inputs(rows, d, f, dtype)
    _, ab = forward(x, w, bias, act)
    for at, columns in ((rows - 1, CLOSED), (1, OPEN)):
        bad = dh.clone()
        bad[at, columns] = value
        none = columns + [f + c for c in columns]
        for kept in (None, ab):
            none_at(backward(x, w, bias, kept, bad, act), backward(x, w, bias, kept, torch.where(torch.isfinite(bad), bad, 0.0), act), [at], none)


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,f", SIZES)
def test_values_that_are_not_finite_behind_closed_gates(rows, d, f, dtype, act):
    x, w, bias, dh = inputs(rows, d, f, dtype)
    wide = bias.clone()
    wide[f + CLOSED[1]] = float("inf")
    h, ab = forward(x, w, wide, act)
    assert torch.isnan(h[:, CLOSED[1]]).all()
    clean = backward(x, w, bias, None, dh, act)
    for kept in (None, ab):
        dx, dw, db = backward(x, w, wide, kept, dh, act)
        assert not torch.isfinite(dx).any()
        mask = torch.zeros(2 * f, dtype=torch.bool, device="cuda")
        mask[CLOSED[1]] = True                # of the gate alone: its value's gradient is dh act(a) = 0
        assert not torch.isfinite(dw[mask]).any() and not torch.isfinite(db[mask]).any()
        assert torch.isfinite(dw[~mask]).all() and torch.isfinite(db[~mask]).all()
        if kept is None:
            assert torch.equal(dw[~mask], clean[1][~mask]) and torch.equal(db[~mask], clean[2][~mask])


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,f", SIZES)
def test_gates_of_minus_infinity(rows, d, f, dtype, act):
    x, w, bias, dh = inputs(rows, d, f, dtype)
    shut = bias.clone()
    shut[CLOSED[0]] = -float("inf")
    h, ab = forward(x, w, shut, act)
    assert (h[:, CLOSED[0]] == 0).all() and torch.isfinite(h).all()
    for kept in (None, ab):
        got = backward(x, w, shut, kept, dh, act)
        assert all(torch.isfinite(v).all() for v in got)
        assert not got[1][CLOSED[0]].any() and not got[1][f + CLOSED[0]].any() and got[2][CLOSED[0]] == 0 and got[2][f + CLOSED[0]] == 0
