"""Gradient clipping inside the training iteration, against the gradients that the iteration leaves (acc_get_grads) in 64 bits.

Tolerances.  The norm is a sum of exact squares in fp64, rounded once: 2^-24 relative, and the quotient of the factor another 2^-24.  An updated weight is
w - lr * (g f) with g f rounded to fp32 and the rest rounded once: half a step of the weight, and of what is taken from it 2^-24 for g f and 2 * 2^-24 for f."""
import ctypes as C

import numpy as np
import pytest

import synth as S

MiB = 1 << 20
U = 2.0 ** -24


def B():
    from paper_1901_06773_amd import binding
    return binding


def small():
    return S.resnet((1, 2), in_hw=32, classes=10, width=8)


def context(net, dtype=0, clip=None, graph=False, mode=None, budget=256 * MiB, k=3):
    b = B()
    ctx = b.Context(net.as_array(), (net.in_c, net.in_h, net.in_w), pool_bytes=budget, host_bytes=64 * MiB, dtype=dtype)
    ctx.set_weights(S.init_params(net))
    ctx.plan_swaps(k, budget, b.PLAN_NONE if mode is None else mode)
    if graph:
        ctx.set_graph(True)
    if clip is not None:
        ctx.set_grad_clip(clip)
    return ctx


def step(ctx, net, s, k=3, lr=0.1):
    import torch
    img, lab = S.make_batch(net, k, s)
    before = ctx.get_weights()
    loss = ctx.train_step(torch.from_numpy(img).pin_memory(), lab, lr)
    return loss, before, ctx.get_grads(), ctx.get_weights()


def norm_of(grads):
    return float(np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads)))


def check(before, grads, after, lr, bound):
    n = norm_of(grads)
    f = 1.0 if n <= bound else bound / n
    for w, g, v in zip(before, grads, after):
        w, g, v = (t.astype(np.float64) for t in (w, g, v))
        taken = lr * f * g
        assert (np.abs(v - (w - taken)) <= U * np.abs(w - taken) + 4 * U * np.abs(taken) + 1e-40).all()
    return n


def same(a, b):
    return all(np.array_equal(x.view(np.uint32), y.view(np.uint32)) for x, y in zip(a, b))


@pytest.mark.gpu
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("dtype", [0, 1])
def test_the_update_takes_the_scaled_gradient(dtype, graph):
    net = small()
    ctx = context(net, dtype, clip=0.05, graph=graph)
    lr = float(np.float32(0.1))
    for s in range(4):                          # (with a graph: recorded, then replayed)
        loss, before, grads, after = step(ctx, net, s)
        n = check(before, grads, after, lr, float(np.float32(0.05)))
        assert np.isfinite(loss) and n > 0.05 and abs(ctx.grad_norm() / n - 1) <= 2 * U
    ctx.set_grad_clip(0)
    loss, before, grads, after = step(ctx, net, 4)
    check(before, grads, after, lr, np.inf)
    with pytest.raises(B().AccError):
        ctx.grad_norm()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("bound", [1e9, float("inf")])
def test_a_bound_that_is_not_reached_changes_nothing(bound):
    net = small()
    plain, clipped = context(net), context(net, clip=bound)
    for s in range(2):
        a, b = step(plain, net, s), step(clipped, net, s)
        assert a[0] == b[0] and same(a[2], b[2]) and same(a[3], b[3])
        assert abs(clipped.grad_norm() / norm_of(b[2]) - 1) <= 2 * U
    plain.close()
    clipped.close()


@pytest.mark.gpu
def test_swapped_and_poisoned_iterations_take_the_same_steps():
    net = small()
    b = B()
    resident, swapped = context(net, clip=0.05), context(net, clip=0.05, mode=b.PLAN_NAIVE_ALL)
    swapped.set_debug(True)
    for s in range(3):
        x, y = step(resident, net, s), step(swapped, net, s)
        assert x[0] == y[0] and same(x[2], y[2]) and same(x[3], y[3]) and resident.grad_norm() == swapped.grad_norm()
    resident.close()
    swapped.close()


def test_refusals():
    b = B()
    lib = b.lib()
    net = small()
    ctx = b.Context(net.as_array(), (net.in_c, net.in_h, net.in_w))          # no device
    for bad in (-1.0, float("nan"), float("-inf")):
        with pytest.raises(b.AccError) as e:
            ctx.set_grad_clip(bad)
        assert e.value.status == b.ACC_EINVAL
    with pytest.raises(b.AccError):
        ctx.set_grad_clip(1.0)
    with pytest.raises(b.AccError):
        ctx.grad_norm()
    assert lib.acc_set_grad_clip(None, 1.0) == b.ACC_EINVAL and "acc_set_grad_clip" in lib.acc_last_error(None).decode()
    assert lib.acc_get_grad_norm(None, C.byref(C.c_float())) == b.ACC_EINVAL
    ctx.close()
