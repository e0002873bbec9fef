"""Distillation at high temperatures, where teacher and student are nearly alike and T^2 stands before what little sets them apart.

With x_j = (t_j - t_max) - (z_j - z_max) of a list that holds every class, p its probabilities and x' what lies about the mean of x, T^2 KL is
T^2 log sum p e^(-x' / T) = sum p x'^2 / 2 (1 + O(x' / T)) and T (q - p) is T p (e^(-x' / T - KL) - 1).

Tolerances.  Four roundings of 2^-24 of the logits' range R leave x' off by 2^-22 R.  A probability is known to 2^-20 of itself (exponents below 16: 16
roundings of 2^-24 of one, and a few of the sum and the quotient), and so is what is left to the unlisted classes.  So T^2 KL is off by sum p |x'| 2^-22 R <=
2^-22 R (2 T^2 KL)^(1/2), doubled for the higher terms, and 2^-18 of itself; T (q - p) by 2^-21 R and 2^-18 of T (q - p) / p times the larger of p and q; a bf16
result by its own rounding, 2^-8 of it, besides.

The reference, in 64 bits, works by differences, too; at the highest temperatures the limit, half the variance of x, stands beside it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def B():
    from paper_1901_06773_amd import binding
    return binding


def inputs(n, classes, k, dtype, seed=1):
    """Lists of the k largest of the teacher's logits in no order; a student that is not far from it."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    teacher = torch.randn(n, classes, generator=g, device="cuda")
    top, index = torch.topk(teacher, k, dim=1)
    order = torch.argsort(torch.rand(n, k, generator=g, device="cuda"), 1)
    z = (0.7 * teacher + torch.randn(n, classes, generator=g, device="cuda")).to(DT[dtype])
    labels = torch.randint(classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    return z, index.gather(1, order).to(torch.int32).contiguous(), top.gather(1, order).contiguous(), labels


def call(z, index, top, labels, temperature, alpha, inplace=False):
    n, classes = z.shape
    nan = float("nan")
    rows, loss, dz = torch.full((n,), nan, device="cuda"), torch.full((1,), nan, device="cuda"), z.clone() if inplace else torch.full_like(z, nan)
    ws = torch.full((B().op_distill_workspace(n, classes, index.shape[1], B()._dtype_of(z)),), 255, dtype=torch.uint8, device="cuda")
    B().op_distill(dz if inplace else z, index, top, labels, rows, loss, dz, temperature, alpha, ws)
    return rows, loss, dz


def reference(z, index, top, temperature):
    """T^2 KL, T (q - p) and the larger of p and q, of the teacher alone; R.  By differences, which 64 bits hold at any temperature."""
    z, top, at = z.double(), top.double(), index.long()
    n, classes = z.shape
    p = torch.softmax(top / temperature, 1)
    x = (top - top.max(1, keepdim=True).values) - (z.gather(1, at) - z.max(1, keepdim=True).values)
    mean = (p * x).sum(1, keepdim=True)
    y = (x - mean) / temperature
    phi = torch.where(y.abs() < 1e-3, y * y * (0.5 - y / 6 + y * y / 24), torch.expm1(-y) + y)
    unlisted = torch.ones_like(z).scatter_(1, at, 0.0)
    e = torch.exp((z - z.max(1, keepdim=True).values) / temperature)
    total = torch.exp((top - top.max(1, keepdim=True).values) / temperature).sum(1, keepdim=True)
    rest = (e * unlisted).sum(1, keepdim=True) * torch.exp(mean / temperature) / total
    kl = torch.log1p((p * phi).sum(1, keepdim=True) + rest)
    q = e / e.sum(1, keepdim=True)
    dz = temperature * q * unlisted
    dz.scatter_(1, at, temperature * p * torch.expm1(-y - kl))
    large = q.scatter(1, at, torch.maximum(p, q.gather(1, at)))
    reach = (top.max(1).values - top.min(1).values) + (z.max(1).values - z.min(1).values)
    return temperature ** 2 * kl.view(n), dz, large, reach


def agree(got, ref, dtype, alpha, hard=None):
    loss, dz, large, reach = ref
    n = len(loss)
    loss, dz = alpha * loss, alpha * dz
    off = 2.0 ** -21 * reach * alpha * (2 * loss / alpha).abs().sqrt() + 2.0 ** -18 * loss.abs()
    grad_off = alpha * 2.0 ** -21 * reach[:, None] * large + 2.0 ** -18 * dz.abs()
    if hard is not None:
        loss, dz, off, grad_off = loss + hard[0], dz + hard[1], off + 2e-5 * (1 + hard[0].abs()), grad_off + 2e-5 * (hard[1].abs() + hard[2])
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    assert all(torch.isfinite(v).all() for v in got)
    assert ((got[0].double() - loss).abs() <= off).all(), float(((got[0].double() - loss).abs() / loss.abs()).max())
    assert abs(float(got[1]) - float(loss.mean())) <= float(off.mean()) + 2.0 ** -23 * abs(float(loss.mean()))
    wrong = (got[2].double() * n - dz).abs() - grad_off - half * (dz.abs() + grad_off) - 1e-37
    assert (wrong <= 0).all(), (float(wrong.max()), int(wrong.argmax()))


TEMPERATURES = [5.0, 20.0, 100.0, 1000.0, 1e4]
# a wave and a workgroup per row of each size, rows that are cut, few and many
SIZES = [(3, 2, 2), (5, 10, 10), (2000, 10, 10), (7, 100, 100), (3000, 100, 64), (41, 1000, 1000), (6, 1021, 1021), (9, 1024, 1000), (2, 1023, 1024 - 3), (65, 300, 299)]


@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", SIZES)
def test_lists_of_all_classes_and_nearly_all(n, classes, k, dtype, temperature):
    z, index, top, labels = inputs(n, classes, k, dtype)
    got = call(z, index, top, None, temperature, 1.0)
    ref = reference(z, index, top, temperature)
    agree(got, ref, dtype, 1.0)
    again = call(z, index, top, None, temperature, 1.0, inplace=True)
    assert all(torch.equal(u, v) for u, v in zip(got, again))
    # a label beside it
    s = torch.log_softmax(z.double(), 1)
    one = torch.zeros_like(s).scatter_(1, labels.long()[:, None], 1.0)
    hard = (-0.25 * (s * one).sum(1), 0.25 * (torch.exp(s) - one), 0.25 * (torch.exp(s) + one))
    agree(call(z, index, top, labels, temperature, 0.75), ref, dtype, 0.75, hard)


@pytest.mark.parametrize("temperature", [1e9, 1e12, 1e18])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes", [(3, 2), (5, 10), (2000, 10), (41, 1000), (6, 1021)])
def test_the_limit_of_high_temperatures(n, classes, dtype, temperature):
    z, index, top, _ = inputs(n, classes, classes, dtype)
    got = call(z, index, top, None, temperature, 1.0)
    agree(got, reference(z, index, top, temperature), dtype, 1.0)
    x = top.double() - z.double().gather(1, index.long())
    variance = ((x - x.mean(1, keepdim=True)) ** 2).mean(1) / 2
    assert ((got[0].double() - variance).abs() <= 1e-4 * variance).all()


@pytest.mark.parametrize("temperature", [5.0, 30.0, 1000.0, 1e6])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(3, 3000, 1024), (40, 5003, 1024), (9, 30001, 1000), (3, 33591, 1024), (5, 300007, 1024), (2, 1 << 20, 700)])
def test_long_rows_of_which_all_but_the_list_is_ruled_out(n, classes, k, dtype, temperature):
    # the student has ruled out what the list doesn't hold, but for three classes far below: what they have stands against little
    z, index, top, _ = inputs(n, classes, k, dtype)
    unlisted = torch.ones(n, classes, dtype=torch.bool, device="cuda").scatter_(1, index.long(), False)
    z[unlisted] = -float("inf")
    free = unlisted.int().argmax(1)
    for low in (1e30, 6 * temperature):
        z[torch.arange(n, device="cuda"), free] = torch.tensor(-low, device="cuda").to(z.dtype)
        ref = reference(z, index, top, temperature)
        ref = ref[:3] + (top.max(1).values.double() - top.min(1).values + (z.gather(1, index.long()).double().max(1).values - z.gather(1, index.long()).double().min(1).values),)
        agree(call(z, index, top, None, temperature, 1.0), ref, dtype, 1.0)


@pytest.mark.parametrize("temperature", [8.0, 200.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(5, 30, 30), (4, 700, 700), (6, 2000, 1024), (3, 40000, 20), (3, 300007, 50)])
def test_entries_without_probability_twice_listed_and_beyond(n, classes, k, dtype, temperature):
    z, index, top, _ = inputs(n, classes, k, dtype)
    top[0, 1:k // 2] = -float("inf")                   # ruled out by the teacher: the student's probability is the gradient
    got = call(z, index, top, None, temperature, 1.0)
    p, q = torch.softmax(top.double() / temperature, 1), torch.softmax(z.double() / temperature, 1)
    ref = temperature * q[0, index[0, 1:k // 2].long()] / n
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    assert ((got[2][0, index[0, 1:k // 2].long()].double() - ref).abs() <= (half + 2.0 ** -18) * ref).all()
    assert torch.isfinite(got[0]).all()
    index[1, 0] = index[1, k - 1]                      # twice
    got = call(z, index, top, None, temperature, 1.0)
    at = int(index[1, 0])
    ref = temperature * (q[1, at] - p[1, 0] - p[1, k - 1]) / n
    size = temperature * (q[1, at] + p[1, 0] + p[1, k - 1]) / n
    assert abs(float(got[2][1, at]) - float(ref)) <= 2.0 ** -18 * float(size) + half * abs(float(ref))
    rows = temperature ** 2 * (p * (torch.log(p) - torch.log(q).gather(1, index.long())))[1].sum()
    assert abs(float(got[0][1]) - float(rows)) <= 2.0 ** -18 * temperature ** 2 * 12
    index[2, 3] = classes                              # no such class
    got = call(z, index, top, None, temperature, 1.0)
    assert torch.isnan(got[0][2]) and torch.isfinite(got[2]).all()
    z[2, 1] = float("nan")
    got = call(z, index, top, None, temperature, 1.0)
    assert torch.isnan(got[2][2]).all() and torch.isfinite(got[2][:2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(7, 100, 100), (41, 1000, 1000), (3, 40000, 64), (4, 300007, 30)])
def test_replayed_at_a_high_temperature(n, classes, k, dtype):
    z, index, top, _ = inputs(n, classes, k, dtype)
    rows, loss, dz = torch.empty(n, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(z)
    ws = torch.empty(B().op_distill_workspace(n, classes, k, B()._dtype_of(z)), dtype=torch.uint8, device="cuda")
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        B().op_distill(z, index, top, None, rows, loss, dz, 50.0, 1.0, ws)
    for seed in (2, 3, 4):
        for a, b in zip((z, index, top), inputs(n, classes, k, dtype, seed)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = call(z, index, top, None, 50.0, 1.0)
        assert torch.equal(got[0], rows) and torch.equal(got[1], loss) and torch.equal(got[2], dz)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_both_sides_of_the_temperature_that_divides_the_ways(dtype):
    z, index, top, _ = inputs(64, 500, 500, dtype)
    below, above = (call(z, index, top, None, t, 1.0) for t in (4.0, 4.000001))
    assert ((below[0] - above[0]).abs() <= 2e-4 * above[0]).all()
    assert (below[2].float() - above[2].float()).norm() <= (2.0 ** -8 if dtype == "bf16" else 1e-4) * above[2].float().norm()
