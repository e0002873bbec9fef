"""Convolution, group norm with its activation, pooling, the linear cross-entropy, their gradients and the clipping of these, one behind the
other as a training step uses them, against 64 bits.  Tolerance: the products are those of test_gpu_ops.py (1e-4 of a tensor's norm)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TOL = 1e-4


def B():
    from paper_1901_06773_amd import binding
    return binding


@pytest.mark.parametrize("k,hw,cin,cout,groups,classes,act", [(4, 9, 32, 64, 8, 100, 2), (3, 14, 64, 128, 32, 1000, 1), (1, 7, 32, 96, 3, 5, 0)])
def test_one_training_step(k, hw, cin, cout, groups, classes, act):
    g = torch.Generator(device="cuda").manual_seed(5)

    def randn(*s):
        return torch.randn(*s, generator=g, device="cuda")
    b = B()
    x, w = randn(k, hw, hw, cin), randn(cout, 3, 3, cin) * (2 / (9 * cin)) ** 0.5
    gamma, beta, fw, fb = 1 + 0.1 * randn(cout), 0.1 * randn(cout), randn(classes, cout) * cout ** -0.5, 0.1 * randn(classes)
    labels = torch.randint(classes, (k,), generator=g, device="cuda", dtype=torch.int32)

    c1, y = torch.empty(k, hw, hw, cout, device="cuda"), torch.empty(k, hw, hw, cout, device="cuda")
    mean, istd = torch.empty(k, groups, device="cuda"), torch.empty(k, groups, device="cuda")
    pooled, loss = torch.empty(k, cout, device="cuda"), torch.empty(1, device="cuda")
    gn_ws = torch.empty(b.op_gn_workspace(k, hw * hw, cout, groups), dtype=torch.uint8, device="cuda")
    ce_ws = torch.empty(b.op_linear_ce_workspace(k, cout, classes, True), dtype=torch.uint8, device="cuda")
    cv_ws = torch.empty(b.op_conv_workspace(k, hw, hw, cin, cout, 3, 1, 1), dtype=torch.uint8, device="cuda")
    dpool, dy, dc = torch.empty_like(pooled), torch.empty_like(y), torch.empty_like(y)
    grads = [torch.empty_like(t) for t in (w, gamma, beta, fw, fb)]
    dw, dgamma, dbeta, dfw, dfb = grads

    b.op_conv_fwd(x, w, c1, 1, 1)
    b.op_gn_fwd(c1, gamma, beta, None, y, mean, istd, groups, act, 1e-5, gn_ws)
    b.op_gap_fwd(y, pooled)
    b.op_linear_ce(pooled, fw, fb, labels, None, loss, dpool, dfw, dfb, ce_ws)
    b.op_gap_bwd(dpool, dy)
    b.op_gn_bwd(c1, dy, y if act == 1 else None, None, gamma, beta, mean, istd, dc, dgamma, dbeta, None, groups, act, gn_ws)
    b.op_conv_wgrad(x, dc, dw, 1, 1, cv_ws)
    norm, clipped = torch.empty(1, device="cuda"), [torch.empty_like(t) for t in grads]
    b.op_grad_clip(b.TensorList(grads, clipped), 0.25, norm, torch.empty(b.op_grad_norm_workspace(), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()

    p = [t.double().cpu().requires_grad_() for t in (w, gamma, beta, fw, fb)]
    z = torch.nn.functional.conv2d(x.double().cpu().permute(0, 3, 1, 2), p[0].permute(0, 3, 1, 2), padding=1)
    v = z.reshape(k, groups, -1)
    v = (v - v.mean(2, keepdim=True)) * (v.var(2, unbiased=False, keepdim=True) + 1e-5) ** -0.5
    a = v.view(z.shape) * p[1].view(1, -1, 1, 1) + p[2].view(1, -1, 1, 1)
    a = {0: a, 1: a * (y.cpu().permute(0, 3, 1, 2) > 0), 2: a * torch.sigmoid(a)}[act]
    logits = a.mean((2, 3)) @ p[3].T + p[4]
    ref = (torch.logsumexp(logits, 1) - logits.gather(1, labels.cpu().long()[:, None])[:, 0]).mean()
    ref.backward()
    assert abs(float(loss) - float(ref)) <= TOL * float(ref)
    for name, got, want in zip(("filter", "scale", "shift", "fc", "fc bias"), grads, p):
        assert (got.double().cpu() - want.grad).norm() <= TOL * want.grad.norm(), name
    total = sum(float((t.grad ** 2).sum()) for t in p) ** 0.5
    assert abs(float(norm) - total) <= TOL * total
    for got, want in zip(clipped, p):
        assert (got.double().cpu() - want.grad * min(1.0, 0.25 / total)).norm() <= 2 * TOL * want.grad.norm()
