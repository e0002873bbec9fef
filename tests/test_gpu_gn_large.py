"""Group norm of tensors beyond 4 GiB, in the two launches and in slices: an image has the bits that it has at the start of a tensor, and the parameters' gradients
are the sums over all images.  Tolerances of test_gpu_gn.py."""
import pytest
import torch

import test_gpu_gn as G

pytestmark = pytest.mark.gpu
U = G.U


def bits(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def summed(x, dy, y, mean, istd, groups):
    """dbeta and dgamma in 64 bits, image by image, and the sums of their terms' magnitudes"""
    c = x.shape[-1]
    out = [torch.zeros(c, dtype=torch.float64, device="cuda") for _ in range(4)]
    step = max(1, (1 << 26) // x[0].numel())
    for i in range(0, x.shape[0], step):
        part = slice(i, i + step)
        per = (x[part].shape[0], 1, groups, 1)
        xh = ((G.groups_of(x[part], groups) - mean[part].double().view(per)) * istd[part].double().view(per)).flatten(2)
        g = torch.where(y[part].flatten(1, 2) > 0, dy[part].flatten(1, 2), 0.0).double()
        for t, v in zip(out, (g, g * xh, g.abs(), (g * xh).abs())):
            t += v.sum((0, 1))
    return out


def check(n, hw, c, groups, order, alone):
    """The whole tensor, and the images `order` at the start of another one of `alone` images; all ReLU, bf16."""
    torch.cuda.empty_cache()
    x = torch.empty(n, 1, hw, c, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    assert x.numel() * 2 > 4 << 30
    gamma, beta = 1 + 0.3 * G.randn(2, c), 0.3 * G.randn(3, c)
    y, mean, istd = G.forward(x, gamma, beta, None, groups, 1)
    dy = x.flip(0).contiguous()
    dx, dg, db, _ = G.backward(x, dy, y, None, gamma, beta, mean, istd, groups, 1, False)
    rest = [i for i in range(n) if i not in order][:alone - len(order)]
    pick = torch.tensor(list(order) + rest, device="cuda")
    x2, dy2 = x[pick], dy[pick]
    y2, mean2, istd2 = G.forward(x2, gamma, beta, None, groups, 1)
    dx2, _, _, _ = G.backward(x2, dy2, y2, None, gamma, beta, mean2, istd2, groups, 1, False)
    for at, i in enumerate(order):
        assert torch.equal(mean[i], mean2[at]) and torch.equal(istd[i], istd2[at])
        assert bits(y[i], y2[at]) and bits(dx[i], dx2[at])
    sb, sg, mb, mg = summed(x, dy, y, mean, istd, groups)
    assert ((db.double() - sb).abs() <= 256 * U * mb).all() and ((dg.double() - sg).abs() <= 256 * U * mg).all()
    return x2, dy2, y2, mean2, istd2, dx2, gamma, beta


def test_two_launches():
    check(3, 12_000_000, 64, 32, (2,), 3)       # (as many images, so that their rows are cut alike)
    torch.cuda.empty_cache()


def test_slices():
    n, hw, c, groups = 5600, 784, 512, 32
    x, dy, y, mean, istd, dx, gamma, beta = check(n, hw, c, groups, (n - 1, 0, n // 2), 3)
    G.check_forward(x, gamma, beta, None, groups, 1, 2.0 ** -8)
    G.check_backward(x, dy, y, None, gamma, beta, mean, istd, groups, 1, 2.0 ** -8, False)
    torch.cuda.empty_cache()
