"""Linear cross-entropy of the most rows there may be, and of more values than a launch has threads (2^32): 2^34 values of x and of its gradient.  Tolerances of
test_gpu_linear_ce.py; a sum over n rows is off by 2^-24 n^(1/2) more (roundings at random of partial sums that grow as the root)."""
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


@pytest.mark.parametrize("dtype,d,classes", [("f32", 4, 300), ("bf16", 24, 700), ("bf16", 1032, 70)])
def test_the_most_rows_that_are_taken(dtype, d, classes):
    n = 1 << 20
    torch.cuda.empty_cache()
    x, w, b, labels = T.inputs(n, d, classes, dtype)
    labels[::7] = -1
    got, ref = T.call(x, w, b, labels, ignore=-1), T.reference(x, w, b, labels, ignore=-1)
    for k, v in got.items():
        tol = T.TOL + (2.0 ** -14 if k in ("dw", "db") else 0.0) + (2.0 ** -8 if k == "dx" and dtype == "bf16" else 0.0)
        assert torch.isfinite(v).all() and (v.double() - ref[k]).norm() <= tol * ref[k].norm(), k
    del got, ref, x
    torch.cuda.empty_cache()
