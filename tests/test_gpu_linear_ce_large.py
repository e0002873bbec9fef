"""Linear cross-entropy of more values than a launch has threads (2^32): 2^34 values of x and of its gradient.  Tolerances of test_gpu_linear_ce.py."""
import pytest
import torch

import test_gpu_linear_ce as T

pytestmark = pytest.mark.gpu


def test_a_gradient_of_more_values_than_a_launch_has_threads():
    n, d, classes = 1 << 18, 1 << 16, 2
    torch.cuda.empty_cache()
    need = 6 * n * d * 2 + (4 << 30)            # x, dx, and copies of both in fp32
    if torch.cuda.mem_get_info()[0] < need:
        pytest.skip("needs 200 GiB")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = (2 / d ** 0.5 * torch.randn(classes, d, generator=g, device="cuda")).bfloat16()
    labels = torch.randint(classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    rows, loss, dx = torch.empty(n, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(x)
    ws = torch.empty(T.B().op_linear_ce_workspace(n, d, classes, True, T.B().BF16), dtype=torch.uint8, device="cuda")
    T.B().op_linear_ce(x, w, None, labels, rows, loss, dx, None, None, ws)
    torch.cuda.synchronize()
    for at in (0, n // 2 - 40, n - 64):         # the last ones are those that a smaller launch would not have reached
        part = slice(at, at + 64)
        z = x[part].double() @ w.double().T
        dz = torch.softmax(z, 1)
        dz[torch.arange(64, device="cuda"), labels[part].long()] -= 1.0
        ref = dz @ w.double() / n
        lse = torch.logsumexp(z, 1) - z.gather(1, labels[part].long()[:, None])[:, 0]
        assert (rows[part].double() - lse).norm() <= T.TOL * lse.norm()
        assert (dx[part].double() - ref).norm() <= (2.0 ** -7 + T.TOL) * ref.norm()
    assert abs(float(loss) - float(rows.double().mean())) <= 1e-6
    del x, dx, ws
    torch.cuda.empty_cache()
