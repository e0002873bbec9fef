"""The gated layer at sizes that between them are multiplied by every kind of tile that its rules choose from, with sums whole and in parts, on both sides of
10240 rows; none of them fills its tiles.  Tolerances are those of test_gpu_glu.py; a sum, or a part of one that is cut, has up to 31000 terms, which the matrix
cores add up by four or more: it is off by fewer than 2^-24 (2 (n / 4)^(1/2) + 8) = 1.1e-5 of the sum of their sizes where roundings are at random, of which
those sums of terms of both signs use a small part.

Gradients of a ReLU whose gates are worked out again are held, as norms, to more than the 2e-5 of the others.  A gate of spread 1, the sum of d products that
are added sixteen at a time, is rounded d / 16 times by 2^-24 of about one at most: off by e = 2^-24 d^(1/2) / 4.  So of all gates, whose density at 0 is 0.4, a
share of 0.4 e = 2^-24 d^(1/2) / 10 = s is on the other side of 0 than it should be, and takes or leaves out a whole term da beside the half that are open: (2
s)^(1/2) of the norm of the gradients at the gates (3.7e-4 at d = 137, where one gate alone of 10787 x 2317 is 2.8e-4).  Twice that, for the few that they are.
Values by themselves are held as ever: near 0 the slope is either."""
import pytest
import torch

from test_gpu_glu import backward, check_backward, check_forward, curve, inputs, near, projections, E

pytestmark = pytest.mark.gpu

# What the sizes choose, of gate and value / dx / dw where they have launches of their own.
BF16 = [
    (16665, 26, 33), (21925, 24, 72), (22698, 98, 129), (10253, 24, 24),          # pairs of 128 x 128, 256 x 128, 256 x 256 and 64 x 64, two values
    (65, 24, 8488), (136, 24, 11160), (272, 101, 11027), (577, 24, 11032),        # the same with three; a last round in quarters
    (3000, 1024, 4096), (3001, 1023, 4099), (2049, 2055, 8190), (3500, 1024, 2048), (3503, 1001, 2043),      # layers below 4096 rows
    (66, 2704, 1368), (66, 4094, 1103), (10568, 3400, 24), (10371, 3961, 35), (10289, 1, 1),      # projections in parts, 128 x 128 and 64 x 64
    (24210, 264, 24), (22182, 515, 24), (21882, 525, 102), (65, 2768, 1232), (131, 529, 10802),   # dx: 256, 64 and 128 whole, 128 and 256 in parts
    (1, 258, 12118), (1, 559, 10887), (138, 571, 10981), (6116, 1160, 24), (8646, 708, 33), (2367, 3216, 71),      # dw of three values: 256, 64 and 128 whole, 64, 128 and 256 in parts
    (11269, 707, 33), (18896, 642, 65), (11270, 520, 8144), (11095, 24, 14680), (10762, 569, 11833),      # of two: 128 and 256 in parts, 256, 64 and 128 whole
    (10846, 24, 864), (10787, 137, 2317), (10313, 27, 15504),                     # dx and dw in one launch, either in parts and whole
]
F32 = [(5, 394, 2057), (821, 2579, 34), (1, 3320, 456), (1, 130, 8973), (1090, 3676, 19),      # projections in parts of 32 x 128; dw of 32 x 128 in parts and whole, of 64 x 64; dx of 32 x 128
       (24838, 21, 33), (4419, 683, 33), (1, 197, 6448), (12842, 222, 17), (3266, 67, 517), (17499, 17, 17), (5, 18, 8416), (447, 18, 17)]


def check(rows, d, f, dtype, act, kept):
    x, w, b, dh = inputs(rows, d, f, dtype)
    ab = check_forward(x, w, b, act, dtype)
    if act == "relu":
        check_relu(x, w, b, dh)
    else:
        check_backward(x, w, b, None, dh, act, dtype)
    if kept:
        check_backward(x, w, b, ab, dh, act, dtype)


def check_relu(x, w, bias, dh):
    """bf16, projections worked out again."""
    d, f = x.shape[1], w.shape[0] // 2
    got = backward(x, w, bias, None, dh, "relu", "bf16")
    p, size = projections(x, w, bias)
    a, b, ea, eb, g = *p.chunk(2, 1), *(E * size).chunk(2, 1), dh.double()
    v, s = curve(a, "relu")
    dz = torch.cat([g * b * s, g * v], 1)
    es = torch.where(a.abs() <= ea, 1.0, 0.0)
    err = torch.cat([g.abs() * (eb * (s.abs() + es) + b.abs() * es), g.abs() * (1.1 * ea + 2.0 ** -20 * v.abs())], 1) + 2.0 ** -22 * dz.abs()
    x64, w64 = x.double(), w.double()
    dx, dw, db = dz @ w64, dz.T @ x64, dz.sum(0)
    more = 2 * (2 * 2.0 ** -24 * d ** 0.5 / 10) ** 0.5
    ex = (err + (2.0 ** -16 + E) * dz.abs()) @ w64.abs()
    near(got["dx"], dx, ex + 2.0 ** -8 * (dx.abs() + ex), "dx", 2.0 ** -8 + 2e-5 + more)
    near(got["dw"], dw, (err + (2.0 ** -16 + E) * dz.abs()).T @ x64.abs() + 2.0 ** -24 * dw.abs(), "dw", 2.0 ** -16 + 2e-5 + more)
    near(got["db"], db, err.sum(0) + E * dz.abs().sum(0) + 2.0 ** -24 * db.abs(), "db", 2e-5 + more)


@pytest.mark.parametrize("act", ["silu", "relu"])
@pytest.mark.parametrize("rows,d,f", BF16)
def test_bf16(rows, d, f, act):
    check(rows, d, f, "bf16", act, act == "silu")
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,d,f", F32)
def test_f32(rows, d, f):
    check(rows, d, f, "f32", "silu", True)
