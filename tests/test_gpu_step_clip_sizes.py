"""Gradient clipping inside the training iteration where the norm is joined from many sums: networks of several pieces of 16384 gradients with a ragged tail, and
of more pieces than a launch has workgroups; and the update itself with room for a few sums only.  Tolerances of test_gpu_step_clip.py."""
import ctypes as C

import numpy as np
import pytest

import synth as S
import test_gpu_step_clip as T

pytestmark = pytest.mark.gpu
MiB = 1 << 20


def several_pieces():
    return S.resnet((1, 2), in_hw=32, classes=10, width=32)                                  # 192298: twelve pieces


def more_pieces_than_workgroups():
    return S.vgg(cfg=((16,),), in_hw=8, classes=10, fc=6001)                                 # 37.6 million: 2297 pieces


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("dtype", [0, 1])
def test_several_pieces(dtype, graph):
    net = several_pieces()
    ctx = T.context(net, dtype, clip=0.05, graph=graph)
    lr, bound = float(np.float32(0.1)), float(np.float32(0.05))
    for s in range(3):
        loss, before, grads, after = T.step(ctx, net, s)
        n = T.check(before, grads, after, lr, bound)
        assert np.isfinite(loss) and n > bound and abs(ctx.grad_norm() / n - 1) <= 2 * T.U
    ctx.close()


def test_several_pieces_swapped_and_poisoned():
    net, b = several_pieces(), T.B()
    resident, swapped = T.context(net, clip=0.05), T.context(net, clip=0.05, mode=b.PLAN_NAIVE_ALL)
    swapped.set_debug(True)
    for s in range(2):
        x, y = T.step(resident, net, s), T.step(swapped, net, s)
        assert x[0] == y[0] and T.same(x[2], y[2]) and T.same(x[3], y[3]) and resident.grad_norm() == swapped.grad_norm()
    resident.close()
    swapped.close()


@pytest.mark.parametrize("dtype,graph", [(0, False), (1, True)])
def test_more_pieces_than_workgroups(dtype, graph):
    net = more_pieces_than_workgroups()
    assert S.param_count(net) > 2048 * 16384 and S.param_count(net) % 16384
    ctx = T.context(net, dtype, clip=0.05, graph=graph, budget=1024 * MiB)
    lr, bound = float(np.float32(0.1)), float(np.float32(0.05))
    for s in range(2):
        _, before, grads, after = T.step(ctx, net, s)
        n = T.check(before, grads, after, lr, bound)
        assert n > bound and abs(ctx.grad_norm() / n - 1) <= 2 * T.U
    ctx.close()


@pytest.mark.parametrize("room", [256, 264, 1000, 16384, 1 << 20])
@pytest.mark.parametrize("count", [1, 16385, 5_000_001])
def test_sums_that_fit_the_room(count, room):
    import torch
    f = getattr(T.B().lib(), "_ZN3acc18sgd_update_clippedEPfPKfffmPvS0_S3_mP12ihipStream_t")
    f.restype, f.argtypes = C.c_int, [C.c_void_p] * 2 + [C.c_float] * 2 + [C.c_size_t] + [C.c_void_p] * 3 + [C.c_size_t, C.c_void_p]
    gen = torch.Generator(device="cuda").manual_seed(count)
    w, g = torch.randn(count, generator=gen, device="cuda"), torch.randn(count, generator=gen, device="cuda")
    norm, scratch = torch.zeros(1, device="cuda"), torch.full((room + 64,), 77, dtype=torch.uint8, device="cuda")
    before, lr = w.cpu().numpy(), float(np.float32(0.1))
    n = T.norm_of([g.cpu().numpy()])
    bound = float(np.float32(0.3 * n))
    assert f(w.data_ptr(), g.data_ptr(), lr, bound, count, None, norm.data_ptr(), scratch.data_ptr(), room, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert abs(float(norm) / n - 1) <= 2 * T.U and (scratch[room:] == 77).all()
    T.check([before], [g.cpu().numpy()], [w.cpu().numpy()], lr, bound)
    assert f(w.data_ptr(), g.data_ptr(), lr, bound, count, None, norm.data_ptr(), scratch.data_ptr(), 255, None) != 0
