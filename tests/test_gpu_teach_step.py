"""A learning step as the operators are used together: group norm, a gated layer, the pool and a linear layer make a student's logits, which learn from the
top logits of a teacher and from labels; gradients all the way back, clipped.  Against the same formulas in 64 bits.

Tolerance: each of the operators is held to 2e-5 of what it makes (see their own tests); seven of them one behind the other to 2e-4, as norms over a tensor."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TOL = 2e-4


def B():
    from paper_1901_06773_amd import binding
    return binding


def student(x, p, groups):
    n, h, w, c = x.shape
    v = x.reshape(n, h * w, groups, c // groups)
    mean = v.mean((1, 3), keepdim=True)
    var = ((v - mean) ** 2).mean((1, 3), keepdim=True)
    y = ((v - mean) / torch.sqrt(var + 1e-5)).reshape(n, h * w, c) * p["gamma"] + p["beta"]
    a, b = (y @ p["w"].T + p["bias"]).chunk(2, -1)
    return (a * torch.sigmoid(a) * b).mean(1) @ p["head"].T


@pytest.mark.parametrize("kept", [True, False])
@pytest.mark.parametrize("n,h,c,groups,f,classes,k", [(4, 5, 32, 8, 48, 60, 7), (6, 7, 64, 16, 96, 1000, 16), (33, 3, 24, 3, 20, 12, 3)])
def test_one_step(n, h, c, groups, f, classes, k, kept):
    g = torch.Generator(device="cuda")
    g.manual_seed(11)

    def r(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    dev, t, alpha = dict(device="cuda"), 2.0, 0.7
    x, teacher = r(n, h, h, c), 2 * r(n, classes)
    p = dict(gamma=1 + 0.1 * r(c), beta=0.1 * r(c), w=r(2 * f, c) / c ** 0.5, bias=0.1 * r(2 * f), head=r(classes, f) / f ** 0.5)
    labels = torch.randint(classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    labels[-1] = -1                                     # padding
    b = B()

    def ws(size):
        return torch.full((max(size, 16),), 255, dtype=torch.uint8, device="cuda")
    # the teacher's answers
    index, top = torch.empty(n, k, dtype=torch.int32, **dev), torch.empty(n, k, **dev)
    b.op_top_logits(teacher, index, top, None)
    # forward
    y, mean, istd = torch.empty_like(x), torch.empty(n, groups, **dev), torch.empty(n, groups, **dev)
    gn_ws = ws(b.op_gn_workspace(n, h * h, c, groups))
    b.op_gn_fwd(x, p["gamma"], p["beta"], None, y, mean, istd, groups, b.ACT_NONE, 1e-5, gn_ws)
    hid, ab = torch.empty(n, h, h, f, **dev), torch.empty(n, h, h, 2 * f, **dev) if kept else None
    rows = n * h * h
    b.op_glu_fwd(y, p["w"], p["bias"], hid, ab, b.ACT_SILU, ws(b.op_glu_workspace(rows, c, f, False)))
    pooled, z = torch.empty(n, f, **dev), torch.empty(n, 1, 1, classes, **dev)
    b.op_gap_fwd(hid, pooled)
    head = p["head"].view(classes, 1, 1, f)
    b.op_conv_fwd(pooled.view(n, 1, 1, f), head, z, 1, 0)
    # loss and gradients
    loss_rows, loss = torch.empty(n, **dev), torch.empty(1, **dev)
    z2 = z.view(n, classes)
    b.op_distill(z2, index, top, labels, loss_rows, loss, z2, t, alpha, ws(b.op_distill_workspace(n, classes, k)), ignore=-1)
    conv_ws = ws(b.op_conv_workspace(n, 1, 1, f, classes, 1, 1, 0))
    dhead, dpooled = torch.empty_like(head), torch.empty(n, 1, 1, f, **dev)
    b.op_conv_wgrad(pooled.view(n, 1, 1, f), z, dhead, 1, 0, conv_ws)
    b.op_conv_dgrad(z, head, dpooled, 1, 0, conv_ws)
    dhid, dy, dw, db = torch.empty_like(hid), torch.empty_like(y), torch.empty_like(p["w"]), torch.empty(2 * f, **dev)
    b.op_gap_bwd(dpooled.view(n, f), dhid)
    b.op_glu_bwd(y, p["w"], p["bias"], ab, dhid, dy, dw, db, b.ACT_SILU, ws(b.op_glu_workspace(rows, c, f, True)))
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(c, **dev), torch.empty(c, **dev)
    b.op_gn_bwd(x, dy, None, None, p["gamma"], p["beta"], mean, istd, dx, dgamma, dbeta, None, groups, b.ACT_NONE, gn_ws)
    got = dict(gamma=dgamma, beta=dbeta, w=dw, bias=db, head=dhead.view(classes, f))
    norm = torch.empty(1, **dev)
    whole = {a: v.clone() for a, v in got.items()}
    tensors = b.TensorList(list(got.values()))
    b.op_grad_clip(tensors, 0.01, norm, ws(b.op_grad_norm_workspace()))
    # the same in 64 bits
    q = {a: v.double().requires_grad_() for a, v in p.items()}
    x64 = x.double().requires_grad_()
    logits = student(x64, q, groups)
    best = torch.topk(teacher, k, dim=1)
    assert torch.equal(best.values, top) and torch.equal(teacher.gather(1, index.long()), top)
    pt = torch.softmax(top.double() / t, 1)
    lq = torch.log_softmax(logits / t, 1).gather(1, index.long())
    rows64 = alpha * t * t * (pt * (torch.log(pt) - lq)).sum(1)
    kept_rows = labels >= 0
    rows64 = rows64 - (1 - alpha) * torch.log_softmax(logits, 1)[torch.arange(n, device="cuda"), labels.clamp(min=0).long()]
    ref = rows64[kept_rows].sum() / kept_rows.sum()
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) <= TOL * abs(float(ref.detach()))
    assert (dx.double() - x64.grad).norm() <= TOL * x64.grad.norm()
    for a, v in whole.items():
        assert (v.double() - q[a].grad).norm() <= TOL * q[a].grad.norm(), a
    total = sum(float((v.grad ** 2).sum()) for v in q.values()) ** 0.5
    assert abs(float(norm) - total) <= TOL * total
    for a, v in got.items():
        want = q[a].grad * min(1.0, 0.01 / total)
        assert (v.double() - want).norm() <= 2 * TOL * want.norm(), a
