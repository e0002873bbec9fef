"""Group norm, the linear cross-entropy and gradient clipping on two streams at once, each call with a workspace of its own: the bits of calls one after the other."""
import pytest
import torch

import test_gpu_gn as G
import test_gpu_linear_ce as T

pytestmark = pytest.mark.gpu


def both_ways(calls):
    alone = [call() for call in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(4):
        together = []
        for s, call in zip(streams, calls):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                together.append(call())
        torch.cuda.synchronize()
        for a, b in zip(alone, together):
            assert all(torch.equal(p, q) for p, q in zip(a, b) if p is not None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_cross_entropy(dtype):
    def make(n, d, classes):
        x, w, b, labels = T.inputs(n, d, classes, dtype)
        return lambda: list(T.call(x, w, b, labels).values())
    both_ways([make(600, 512, 9000), make(777, 1160, 5001), make(41, 256, 1000)])


@pytest.mark.parametrize("n,hw,c,groups", [(40, 784, 512, 32), (2, 9000, 64, 8)])
def test_group_norm(n, hw, c, groups):
    def make(seed):
        x, dy, gamma, beta = G.randn(seed, n, 1, hw, c), G.randn(seed + 1, n, 1, hw, c), G.randn(seed + 2, c), G.randn(seed + 3, c)

        def call():
            y, mean, istd = G.forward(x, gamma, beta, None, groups, 1)
            return [y, mean, istd, *G.backward(x, dy, y, None, gamma, beta, mean, istd, groups, 1, True)]
        return call
    both_ways([make(1), make(11)])


def test_clipping():
    b = T.B()

    def make(seed):
        tensors = [T.randn(seed + i, k) for i, k in enumerate((5, 100000, 3000001))]

        def call():
            outs, norm = [torch.empty_like(t) for t in tensors], torch.empty(1, device="cuda")
            b.op_grad_clip(b.TensorList(tensors, outs), 10.0, norm, torch.empty(b.op_grad_norm_workspace(), dtype=torch.uint8, device="cuda"))
            return [norm, *outs]
        return call
    both_ways([make(1), make(20)])
