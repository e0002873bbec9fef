"""Group norm where slices of 32 bytes of channels stay in registers (176 to 256 of them) and beside those sizes, against the formulas in 64 bits; tolerances of
test_gpu_gn.py."""
import pytest
import torch

import test_gpu_gn as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,residual", [(0, True), (1, False), (1, True), (2, False), (2, True)])
@pytest.mark.parametrize("n,h,w,c,groups,dtype", [
    (11, 55, 55, 128, 16, "f32"), (16, 55, 55, 128, 16, "f32"), (17, 55, 55, 128, 16, "f32"), (32, 56, 56, 64, 32, "f32"), (12, 56, 56, 256, 32, "bf16"),
    (16, 80, 80, 256, 32, "bf16"), (19, 80, 81, 64, 8, "f32"), (23, 57, 53, 128, 16, "bf16")])
def test_against_the_formulas(n, h, w, c, groups, dtype, act, residual):
    td, hs = G.DT[dtype]
    x = (G.randn(1, n, h, w, c) * (0.5 + 0.1 * G.randn(2, c).abs()) + G.randn(3, c)).to(td)
    gamma, beta = 1 + 0.3 * G.randn(4, c), 0.3 * G.randn(5, c)
    res = G.randn(6, n, h, w, c).to(td) if residual else None
    y, mean, istd = G.check_forward(x, gamma, beta, res, groups, act, hs)
    G.check_backward(x, G.randn(7, n, h, w, c).to(td), y, res, gamma, beta, mean, istd, groups, act, hs, residual)
    torch.cuda.empty_cache()
