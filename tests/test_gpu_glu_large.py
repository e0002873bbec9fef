"""The gated layer at its largest: fp32 tensors beyond 4 GiB, and weights of nearly 2^30 values a side, which is the limit, in both types.  As norms, which
test_gpu_glu.py holds to 2e-5, results in bf16 to their rounding of 2^-8 and dw of bf16 operands to 2^-16 besides."""
import pytest
import torch

from test_gpu_glu import backward, curve, forward, inputs, projections

pytestmark = pytest.mark.gpu


def near(got, ref, tol, what):
    assert torch.isfinite(got).all(), what
    assert (got.double() - ref).norm() <= tol * ref.norm() + 1e-30, (what, float((got.double() - ref).norm() / ref.norm()))


def test_offsets_beyond_32_bits_in_fp32():
    rows, d, f = 150000, 16, 4096                       # 4.9 GB of kept projections and of dz
    x, w, b, _ = inputs(rows, d, f, "f32")
    dh = torch.zeros(rows, f, device="cuda")
    at = torch.tensor([0, 1, 70000, 131071, 131072, 131073, 149999], device="cuda")
    dh[at] = torch.randn(len(at), f, device="cuda")
    h, ab = forward(x, w, b, "silu", "f32")
    p, _ = projections(x[at], w, b)
    a, v = p.chunk(2, 1)
    near(h[at], a * torch.sigmoid(a) * v, 2e-5, "h")
    near(ab[at], p, 2e-5, "ab")
    for kept in (ab, None):
        got = backward(x, w, b, kept, dh, "silu", "f32")
        value, slope = curve(a, "silu")
        dz = torch.cat([dh[at].double() * v * slope, dh[at].double() * value], 1)
        near(got["dx"][at], dz @ w.double(), 2e-5, "dx")
        near(got["dw"], dz.T @ x[at].double(), 2e-5, "dw")
        near(got["db"], dz.sum(0), 4e-5, "db")
        assert (got["dx"].abs().sum(1) != 0).sum() == len(at)
        del got


@pytest.mark.parametrize("rows", [3, 70])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,f", [(16384, 65464), (65528, 16361)])
def test_the_largest_weights(d, f, dtype, rows):
    # in pieces of 4096 columns, so that the reference takes little room; the weights' spread is that of inputs()
    g = torch.Generator(device="cuda").manual_seed(1)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    w = torch.empty(2 * f, d, device="cuda", dtype=dt)
    for c in range(0, 2 * f, 4096):
        w[c:c + 4096] = (torch.randn(min(4096, 2 * f - c), d, generator=g, device="cuda") / d ** 0.5).to(dt)
    x, dh, b = torch.randn(rows, d, generator=g, device="cuda").to(dt), torch.randn(rows, f, generator=g, device="cuda").to(dt), 0.3 * torch.randn(2 * f, generator=g, device="cuda")
    p = torch.cat([x.double() @ w[c:c + 4096].double().T for c in range(0, 2 * f, 4096)], 1) + b.double()
    a, v = p.chunk(2, 1)
    value, slope = curve(a, "silu")
    half = 2.0 ** -8 if dtype == "bf16" else 0
    h, ab = forward(x, w, b, "silu", dtype)
    near(h, value * v, half + 2e-5, "h")
    near(ab, p, half + 2e-5, "ab")
    dz = torch.cat([dh.double() * v * slope, dh.double() * value], 1)
    dx = sum(dz[:, c:c + 4096] @ w[c:c + 4096].double() for c in range(0, 2 * f, 4096))
    got = backward(x, w, b, None, dh, "silu", dtype)
    near(got["dx"], dx, half + 2e-5, "dx")
    near(got["db"], dz.sum(0), 2e-5, "db")
    for c in range(0, 2 * f, 4096):
        near(got["dw"][c:c + 4096], dz[:, c:c + 4096].T @ x.double(), 2.0 ** -16 + 2e-5, "dw")
    del got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,f", [(8, 8), (3, 9), (1, 2)])
def test_the_most_rows(d, f, dtype):
    # dh is 0 but in a few thousand rows: gradients' sums over all of them are no longer than those that test_gpu_glu.py holds
    rows = 1 << 24
    x, w, b, dh = inputs(rows, d, f, dtype)
    h, ab = forward(x, w, b, "silu", dtype)
    at = torch.cat([torch.arange(1500, device="cuda"), torch.arange(rows - 1500, rows, device="cuda"), torch.arange(0, rows, 1 << 13, device="cuda")]).unique()
    p, _ = projections(x[at], w, b)
    a, v = p.chunk(2, 1)
    value, slope = curve(a, "silu")
    half = 2.0 ** -8 if dtype == "bf16" else 0
    near(h[at], value * v, half + 2e-5, "h")
    near(ab[at], p, half + 2e-5, "ab")
    assert torch.isfinite(h).all()
    only = torch.zeros_like(dh)
    only[at] = dh[at]
    dz = torch.cat([dh[at].double() * v * slope, dh[at].double() * value], 1)
    got = backward(x, w, b, None, only, "silu", dtype)
    near(got["dx"][at], dz @ w.double(), half + 2e-5, "dx")
    near(got["dw"], dz.T @ x[at].double(), 2.0 ** -16 + 2e-5, "dw")
    near(got["db"], dz.sum(0), 1e-4, "db")
    assert int((got["dx"] != 0).any(1).sum()) <= len(at)
