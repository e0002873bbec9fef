"""How many bits the gradients of the gated layer keep, against 64 bits, where fewer would show.

Tolerances.  A value held as the sum of two bf16 values is off by 2^-16 of itself at most, of three by 2^-24; a result rounded to bf16 by 2^-8 of itself.
Projections and sums add 1e-5 of the magnitudes that are summed (test_gpu_glu.py)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
ACT = {"none": 0, "relu": 1, "silu": 2}


def B():
    from paper_1901_06773_amd import binding
    return binding


def gradients(x, w, bias, ab, dh, act):
    rows, d, f = x.shape[0], x.shape[1], w.shape[0] // 2
    dx, dw, db = torch.empty_like(x), torch.empty(2 * f, d, device="cuda"), torch.empty(2 * f, device="cuda")
    ws = torch.empty(B().op_glu_workspace(rows, d, f, True, B()._dtype_of(x)), dtype=torch.uint8, device="cuda")
    B().op_glu_bwd(x, w, bias, ab, dh, dx, dw, db, ACT[act], ws)
    return dx, dw, db


def dz_of(ab, dh, act):
    a, b = ab.chunk(2, 1)
    s = torch.sigmoid(a)
    value, slope = (a * s, s * (1 + a * (1 - s))) if act == "silu" else (a, torch.ones_like(a))
    return torch.cat([dh.double() * b * slope, dh.double() * value], 1)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("common", [0, 10, 30])
@pytest.mark.parametrize("rows,d,f", [(300, 128, 64), (64, 256, 1000), (777, 520, 3001), (2000, 1032, 500), (4100, 64, 4096), (5000, 1024, 1024), (131, 33, 57)])
def test_what_the_weights_have_in_common_cancels_in_dx(rows, d, f, common, kept):
    # as in front of a normalisation: a row of dh sums to zero.  Values are near 1, so that the gates' gradients sum to little, too
    g = torch.Generator(device="cuda").manual_seed(3)

    def r(*s):
        return torch.randn(*s, generator=g, device="cuda")
    x = r(rows, d).bfloat16()
    w = torch.cat([(r(f, d) + common * r(d)) / d ** 0.5, 0.05 * r(f, d) / d ** 0.5]).bfloat16()
    bias = torch.cat([torch.zeros(f, device="cuda"), torch.ones(f, device="cuda")])
    dh = r(rows, f)
    dh = (dh - dh.mean(1, keepdim=True)).bfloat16()
    ab = x.double() @ w.double().T + bias.double()
    if kept:
        ab = ab.bfloat16()
    dx = gradients(x, w, bias, ab if kept else None, dh, "none")[0]
    dz = dz_of(ab.double(), dh, "none")
    ref, summed = dz @ w.double(), dz.abs() @ w.double().abs()
    assert (dx.double() - ref).norm() <= 2.0 ** -8 * ref.norm() + (2.0 ** -16 + 1e-5) * summed.norm()


@pytest.mark.parametrize("rows", [1000, 4095, 4096, 6000, 8192, 10239])
@pytest.mark.parametrize("d,f", [(64, 40), (256, 136), (512, 1024)])
def test_dw_keeps_the_digits_of_a_sum_in_fp32(rows, d, f):
    # The running sum of n terms at random is on average n / 2 terms' squares; rounded by 2^-24 of itself at most each time that a product of sixteen terms of
    # one of three values is added, 3 n / 16 times, it is off by (3 n / 32)^(1/2) 2^-24 of the result, as norms.  dz of kept projections is off by a few
    # roundings of 2^-24 and the activation's 2^-22: 4e-7.
    g = torch.Generator(device="cuda").manual_seed(rows + d)

    def r(*s):
        return torch.randn(*s, generator=g, device="cuda")
    x, w, dh, ab = r(rows, d).bfloat16(), (r(2 * f, d) / d ** 0.5).bfloat16(), r(rows, f).bfloat16(), r(rows, 2 * f).bfloat16()
    dw = gradients(x, w, None, ab, dh, "silu")[1]
    ref = dz_of(ab.double(), dh, "silu").T @ x.double()
    assert (dw.double() - ref).norm() <= (4e-7 + 2.0 ** -24 * (3 * rows / 32) ** 0.5) * ref.norm()
