"""How many bits the gradients of the linear cross-entropy keep, against 64 bits, where fewer would show.

Tolerances.  A value held as the sum of two bf16 values is off by 2^-16 of itself at most, of three by 2^-24; a result rounded to bf16 by 2^-8 of itself.  Sums and
logits add 2e-5 of the magnitudes that are summed (test_gpu_linear_ce.py)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def B():
    from paper_1901_06773_amd import binding
    return binding


def inputs(n, d, classes, common, seed=3):
    """bf16 operands; the classes' weights have a part in common, `common` times as large as what sets them apart."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*s):
        return torch.randn(*s, generator=g, device="cuda")
    w = 2 / d ** 0.5 * (randn(classes, d) + common * randn(d))
    labels = torch.randint(classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    x = randn(n, d) + w[labels.long()] * torch.rand(n, 1, generator=g, device="cuda") / (1 + common)
    return x.bfloat16(), w.bfloat16(), labels


def gradients(x, w, labels):
    n, d = x.shape
    classes = w.shape[0]
    dx, dw = torch.empty_like(x), torch.empty(classes, d, device="cuda")
    ws = torch.empty(B().op_linear_ce_workspace(n, d, classes, True, B()._dtype_of(x)), dtype=torch.uint8, device="cuda")
    B().op_linear_ce(x, w, None, labels, None, None, dx, dw, None, ws)
    return dx, dw


def dz_of(x, w, labels):
    n = x.shape[0]
    dz = torch.softmax(x.double() @ w.double().T, 1)
    dz[torch.arange(n, device="cuda"), labels.long()] -= 1.0
    return dz / n


@pytest.mark.parametrize("common", [0, 10, 30])
@pytest.mark.parametrize("n,d,classes", [(64, 256, 1000), (300, 128, 10), (256, 1160, 5000), (777, 520, 3001), (4100, 64, 33333), (4100, 1032, 2000)])
def test_what_the_weights_have_in_common_cancels_in_dx(n, d, classes, common):
    x, w, labels = inputs(n, d, classes, common)
    dx, _ = gradients(x, w, labels)
    dz = dz_of(x, w, labels)
    ref, summed = dz @ w.double(), dz.abs() @ w.double().abs()
    assert (dx.double() - ref).norm() <= 2.0 ** -8 * ref.norm() + (2.0 ** -16 + 2e-5) * summed.norm()


# A gradient's sum of up to 2048 products is rounded some 400 times, by 2^-24 of a partial sum that grows as the square root: 2^-24 * (400 / 2 / 3)^(1/2) = 2^-21 of the
# result.  A logit of 8 that is off by a rounding or two moves dz by 2^-21 to 2^-20 of itself.


@pytest.mark.parametrize("n,d,classes", [(64, 256, 1000), (512, 256, 1000), (1000, 512, 4000), (1024, 64, 20000), (777, 1160, 3001)])
def test_dw_of_bf16_operands_keeps_three_values_of_dz(n, d, classes):
    """Three values are within 2^-24 and leave the sums' own error; two are off by 2^-19.5 and more."""
    x, w, labels = inputs(n, d, classes, 0)
    _, dw = gradients(x, w, labels)
    ref = dz_of(x, w, labels).T @ x.double()
    assert (dw.double() - ref).norm() <= 2.0 ** -20 * ref.norm()


@pytest.mark.parametrize("n,d,classes", [(4096, 256, 1000), (5001, 520, 4000)])
def test_dw_of_many_rows_keeps_two_values_of_dz(n, d, classes):
    """Two values are within 2^-16, and 2^-19 as errors at random; one is off by 2^-10."""
    x, w, labels = inputs(n, d, classes, 0)
    _, dw = gradients(x, w, labels)
    ref = dz_of(x, w, labels).T @ x.double()
    assert (dw.double() - ref).norm() <= 2.0 ** -18 * ref.norm()


@pytest.mark.parametrize("n,d,classes", [(1024, 1024, 8192), (2048, 512, 20000), (1000, 515, 9001), (600, 512, 30000), (777, 1160, 5000)])
def test_fp32_products_on_the_bf16_matrix_cores_keep_three_values(n, d, classes):
    """Sizes of 128 x 128 tiles in all three products.  An fp32 value held as two bf16 values instead of three leaves 2^-17 of a sum (6.9e-6)."""
    x, w, labels = inputs(n, d, classes, 0)
    g = torch.Generator(device="cuda").manual_seed(8)
    x = x.float() + 2.0 ** -9 * torch.rand(n, d, generator=g, device="cuda")       # (all 24 bits)
    w = w.float() * (1 + 2.0 ** -9 * torch.rand(classes, d, generator=g, device="cuda"))
    dx, dw = gradients(x, w, labels)
    dz = dz_of(x, w, labels)
    for got, ref in ((dx, dz @ w.double()), (dw, dz.T @ x.double())):
        assert (got.double() - ref).norm() <= 2.0 ** -18 * ref.norm()


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,classes", [(9, 64, 100), (300, 256, 1500), (1024, 512, 8192), (600, 512, 30000)])
def test_a_row_that_is_not_finite_has_no_finite_loss_and_leaves_the_others(n, d, classes, dtype, value):
    x, w, labels = (t if t.dtype == torch.int32 else t.to(dtype) for t in inputs(n, d, classes, 0))

    def losses():
        rows = torch.empty(n, device="cuda")
        ws = torch.empty(B().op_linear_ce_workspace(n, d, classes, False, B()._dtype_of(x)), dtype=torch.uint8, device="cuda")
        B().op_linear_ce(x, w, None, labels, rows, None, None, None, None, ws)
        return rows
    whole = losses()
    x[5, d // 2] = value
    rows = losses()
    assert torch.isfinite(whole).all() and not torch.isfinite(rows[5])
    others = torch.arange(n, device="cuda") != 5
    assert torch.equal(rows[others], whole[others])
