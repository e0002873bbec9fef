"""Distillation from a teacher's top logits against its formulas in 64 bits.

Tolerances.  An exponent (z - max) / T is off by three roundings of 2^-24 of it, an exponential by that and three of its own, the sum and the
quotient by as many: below an exponent of -40 a probability counts for nothing beside those of the row, so each is known to 2^-24 (3 * 40 + 10) = 8e-6 of
itself, and to 2e-5 with the sum of up to 2^20 of them.  A gradient is made of two to four such terms: it is held to 2e-5 of their sizes, and in bf16 to its own
rounding, 2^-8 of it, besides.  Where exponentials fall under the smallest fp32 value, 1e-37 is lost.  A loss is a sum of terms known to 2e-5 of their sizes."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = 2e-5


def B():
    from paper_1901_06773_amd import binding
    return binding


def inputs(n, classes, k, dtype, seed=1, ragged=False, padded=False, labels=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    teacher = 2 * torch.randn(n, classes, generator=g, device="cuda")
    teacher.scatter_add_(1, torch.randint(classes, (n, 1), generator=g, device="cuda"), 6 * torch.rand(n, 1, generator=g, device="cuda"))
    top, index = torch.topk(teacher, min(k, classes), dim=1)
    z = (0.7 * teacher + torch.randn(n, classes, generator=g, device="cuda")).to(DT[dtype])
    if k > classes:
        top, index = torch.nn.functional.pad(top, (0, k - classes), value=3.0), torch.nn.functional.pad(index, (0, k - classes), value=-1)
    index = index.to(torch.int32)
    if ragged:
        index = torch.where(torch.arange(k, device="cuda") < torch.randint(1, k + 1, (n, 1), generator=g, device="cuda"), index, -5)
    lab = torch.randint(classes, (n,), generator=g, device="cuda", dtype=torch.int32) if labels else None
    if padded:
        index[::3] = -1
        if labels:
            lab[::3] = -9
    return z, index.contiguous(), top.contiguous(), lab


def call(z, index, top, labels, temperature, alpha, ignore=None, want=("rows", "loss", "dz"), inplace=False):
    n, classes = z.shape
    k = index.shape[1]
    nan = float("nan")
    out = dict(rows=torch.full((n,), nan, device="cuda"), loss=torch.full((1,), nan, device="cuda"), dz=z.clone() if inplace else torch.full_like(z, nan))
    out = {a: v if a in want else None for a, v in out.items()}
    ws = torch.full((B().op_distill_workspace(n, classes, k, B()._dtype_of(z)),), 255, dtype=torch.uint8, device="cuda")
    B().op_distill(out["dz"] if inplace else z, index, top, labels, out["rows"], out["loss"], out["dz"], temperature, alpha, ws, ignore)
    return out


def reference(z, index, top, labels, temperature, alpha, ignore=None):
    """Results, and the sizes of the terms that they are made of."""
    z, top = z.double(), top.double()
    n, classes = z.shape
    every = torch.arange(n, device="cuda")
    there = (index >= 0).long().cumprod(1).bool()
    has = there[:, :1]
    at = torch.where(there, index, 0).long()
    counts = there[:, 0] if labels is None else (labels != ignore if ignore is not None else torch.ones(n, dtype=torch.bool, device="cuda"))
    t = torch.where(there, top / temperature, -torch.inf)
    p = torch.where(there, torch.softmax(torch.where(has, t, 0.0), 1), 0.0)
    log_q = torch.log_softmax(z / temperature, 1)
    log_p = torch.where(p > 0, torch.log(p.clamp(min=1e-320)), 0.0)
    lq = torch.where(p > 0, log_q.gather(1, at), 0.0)
    rows = alpha * temperature ** 2 * (p * (log_p - lq)).sum(1)
    row_size = alpha * temperature ** 2 * ((p * (log_p.abs() + lq.abs())).sum(1) + 1)
    q = torch.exp(log_q) * has
    spread = torch.zeros_like(z).scatter_add_(1, at, p)
    dz, size = alpha * temperature * (q - spread), alpha * temperature * (q + spread)
    if alpha < 1:
        lab = labels.long().clamp(0, classes - 1)
        ls = torch.log_softmax(z, 1)
        rows = rows - (1 - alpha) * ls[every, lab]
        row_size = row_size + (1 - alpha) * (ls[every, lab].abs() + 1)
        s = torch.exp(ls)
        one = torch.zeros_like(z)
        one[every, lab] = 1.0
        dz, size = dz + (1 - alpha) * (s - one), size + (1 - alpha) * (s + one)
    share = counts.double() / max(1, int(counts.sum()))
    rows, row_size = torch.where(counts, rows, 0.0), torch.where(counts, row_size, 0.0)
    dz, size = torch.where(counts[:, None], dz, 0.0), torch.where(counts[:, None], size, 0.0)
    return (dict(rows=rows, loss=(rows * share).sum().view(1), dz=dz * share[:, None]),
            dict(rows=row_size, loss=(row_size * share).sum().view(1), dz=size * share[:, None]))


def agree(got, ref, dtype):
    ref, size = ref
    for what, v in got.items():
        if v is None:
            continue
        half = 2.0 ** -8 if what == "dz" and dtype == "bf16" else 2.0 ** -24
        off = (v.double() - ref[what]).abs() - half * ref[what].abs() - TOL * size[what] - 1e-37
        assert torch.isfinite(v).all(), what
        assert (off <= 0).all(), (what, float(off.max()), int(off.argmax()))


SIZES = [(1, 1, 1), (3, 2, 2), (1, 5, 3), (41, 1000, 16), (64, 1000, 128), (65, 1000, 129), (7, 1021, 5), (300, 10, 10), (1100, 17, 3), (5000, 33, 4), (64, 2039, 64),
         (3, 1500, 1024), (5, 4099, 7), (30, 8191, 70), (130, 9001, 100), (6, 16385, 65), (33, 50001, 37), (9, 65530, 3), (4, 131060, 64), (2, 131072, 64),
         (3, 300007, 100), (1, 1 << 20, 1024), (3, 7, 20), (20001, 9, 3), (1 << 20, 3, 2), (70000, 40, 5)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", SIZES)
def test_against_the_formulas(n, classes, k, dtype):
    for labels, temperature, alpha, ragged in ((False, 2.0, 1.0, False), (True, 4.0, 0.9, True), (True, 1.0, 0.3, False)):
        x = inputs(n, classes, k, dtype, labels=labels, ragged=ragged)
        agree(call(*x, temperature, alpha), reference(*x, temperature, alpha), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(1, 3, 2), (40, 1000, 16), (1030, 100, 7), (25, 5003, 30), (10, 40001, 64), (7, 270001, 20)])
def test_rows_that_do_not_count(n, classes, k, dtype):
    for labels, alpha in ((False, 1.0), (True, 1.0), (True, 0.5)):
        z, index, top, lab = inputs(n, classes, k, dtype, labels=labels, padded=True)
        z[::3] = float("nan")                          # nothing of a padded row is looked at
        got = call(z, index, top, lab, 2.0, alpha, ignore=-9)
        ref = reference(torch.nan_to_num(z), index, top, lab, 2.0, alpha, ignore=-9)
        agree(got, ref, dtype)
        assert (got["rows"][::3] == 0).all() and (got["dz"][::3] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [100, 3001, 30001, 300007])
def test_rows_without_a_list(classes, dtype):
    z, index, top, lab = inputs(12, classes, 9, dtype)
    index[3] = -1
    index[7, 0] = -3                                   # the list ends before its first entry
    agree(call(z, index, top, lab, 2.0, 0.4), reference(z, index, top, lab, 2.0, 0.4), dtype)
    agree(call(z, index, top, None, 2.0, 1.0), reference(z, index, top, None, 2.0, 1.0), dtype)
    index[:] = -1
    got = call(z, index, top, None, 2.0, 1.0)
    assert float(got["loss"]) == 0 and (got["rows"] == 0).all() and (got["dz"] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [50, 3001, 30001, 300007])
def test_classes_listed_twice_and_labels_in_the_list(classes, dtype):
    z, index, top, lab = inputs(10, classes, 40, dtype)
    index[:, 5] = index[:, 0]
    index[:, 39] = index[:, 0]
    index[:, 20:25] = index[:, 30:35]
    lab[:5] = index[:5, 0]
    lab[5:8] = index[5:8, 22]
    for alpha in (1.0, 0.5):
        agree(call(z, index, top, lab, 3.0, alpha), reference(z, index, top, lab, 3.0, alpha), dtype)


@pytest.mark.parametrize("classes", [60, 5001, 40001, 300007])
def test_a_class_that_is_all_but_certain(classes):
    # teacher and student both give it 1 - 1e-6 and less of the rest: the gradient is the difference of the rests
    n, k = 8, 6
    z, index, top, lab = inputs(n, classes, k, "f32")
    every = torch.arange(n, device="cuda")
    best = index[:, 0].long()
    z[every, best] = z.max(1).values + 14 + torch.log(torch.tensor(float(classes)))
    top[:, 0] = top[:, 1] + 15
    lab.copy_(index[:, 0])
    got, (ref, _) = call(z, index, top, lab, 1.0, 0.5), reference(z, index, top, lab, 1.0, 0.5)
    a, r = got["dz"][every, best].double(), ref["dz"][every, best]
    rest = 1 - torch.softmax(top.double(), 1)[:, 0] + 2 * (1 - torch.softmax(z.double(), 1)[every, best])
    assert ((a - r).abs() <= 1e-4 * rest / n).all()    # (of what is left of one, not of one: 6e-8 each)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [40, 2500, 20001, 300007])
def test_values_that_are_not_finite(classes, dtype):
    inf = float("inf")
    z, index, top, lab = inputs(9, classes, 8, dtype)
    top[0, 3] = -inf                                   # a listed class that the teacher rules out
    outside = torch.ones(classes, dtype=torch.bool, device="cuda")
    outside[index[1].long()] = False
    outside[lab[1].long()] = False
    z[1, outside.nonzero().view(-1)[::2]] = -inf       # classes that the student rules out
    top[2, 1:] = -inf                                  # a teacher that is certain
    good = [0, 1, 2, 8]
    z[3, 1] = float("nan")
    z[4, :] = -inf
    top[5, :] = -inf
    index[6, 2] = classes                              # no such class
    lab[7] = classes + 3
    got, ref = call(z, index, top, lab, 2.0, 0.5), reference(torch.nan_to_num(z, nan=0.0, neginf=-1e30), index.clamp(max=classes - 1), torch.nan_to_num(top, neginf=-1e30), lab, 2.0, 0.5)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for r in good:
        assert ((got["dz"][r].double() - ref[0]["dz"][r]).abs() <= half * ref[0]["dz"][r].abs() + TOL * ref[1]["dz"][r] + 1e-37).all(), r
        assert abs(float(got["rows"][r]) - float(ref[0]["rows"][r])) <= TOL * float(ref[1]["rows"][r]), r
    for r in (3, 4, 5, 6, 7):
        assert torch.isnan(got["rows"][r]), r
    for r in (3, 4):
        assert torch.isnan(got["dz"][r]).all(), r
    assert torch.isnan(got["dz"][5, index[5].long()]).all()
    for r in (6, 7):
        assert torch.isfinite(got["dz"][r]).all(), r
    assert torch.isnan(got["loss"]).all()
    z[1, index[1, 0].long()] = -inf                    # a class that the teacher names and the student rules out
    assert call(z, index, top, lab, 2.0, 0.5)["rows"][1] == inf


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(5, 1003, 7), (70, 1003, 140), (9, 20001, 30), (3, 300007, 33)])
def test_in_place_alone_and_again(n, classes, k, dtype):
    x = inputs(n, classes, k, dtype, ragged=True)
    all_of = call(*x, 2.0, 0.7)
    for _ in range(2):
        again = call(*x, 2.0, 0.7, inplace=True)
        assert all(torch.equal(again[w], all_of[w]) for w in again)
    for w in ("rows", "loss", "dz"):
        assert torch.equal(call(*x, 2.0, 0.7, want=(w,))[w], all_of[w]), w


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(5, 1003, 7), (1030, 13, 3), (9, 20001, 30), (3, 300007, 33)])
def test_nothing_is_written_behind_the_results(n, classes, k, dtype):
    z, index, top, lab = inputs(n, classes, k, dtype)
    size = B().op_distill_workspace(n, classes, k, B()._dtype_of(z))
    rows, loss, ws = torch.full((n + 4096,), 77.0, device="cuda"), torch.full((4097,), 77.0, device="cuda"), torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    dz = torch.full((n * classes + 4096,), 77.0, device="cuda", dtype=z.dtype)
    B().op_distill(z, index, top, lab, rows[:n], loss[:1], dz[:n * classes].view(n, classes), 2.0, 0.7, ws[:size])
    assert all((t[-4096:] == 77).all() for t in (rows, loss, ws, dz))
    assert torch.equal(dz[:n * classes].view(n, classes), call(z, index, top, lab, 2.0, 0.7)["dz"])


@pytest.mark.parametrize("labels,alpha", [(False, 1.0), (True, 0.6)])
@pytest.mark.parametrize("classes,k", [(50, 5), (3001, 20), (200003, 20)])
def test_gradient_against_differences(classes, k, labels, alpha):
    # (L(z + h v) - L(z - h v)) / 2 h is off by h^2 / 6 times the third derivative, at most 2 |v|^3 of a row's loss, and by 2^-22 of the loss over h
    z, index, top, lab = inputs(4, classes, k, "f32", labels=labels)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    dz = call(z, index, top, lab, 2.0, alpha)["dz"].double()
    for _ in range(4):
        v, h = torch.zeros_like(z), 2.0 ** -5
        for row in range(4):
            at = index[row, torch.randint(k, (3,), generator=g, device="cuda")].long()
            v[row, at] = torch.sign(torch.randn(3, generator=g, device="cuda"))
        plus, minus = (float(call(z + s * h * v, index, top, lab, 2.0, alpha)["loss"]) for s in (1, -1))
        assert abs((plus - minus) / (2 * h) - float((dz * v).sum())) <= h * h / 6 * 2 * 3 ** 1.5 + 2.0 ** -22 * max(1.0, abs(plus)) * 2 / h


def test_offsets_beyond_32_bits():
    n, classes, k = 2100, 1 << 20, 4                   # 2.2e9 logits
    z = torch.zeros(n, classes, device="cuda", dtype=torch.bfloat16)
    index = (torch.arange(n, device="cuda", dtype=torch.int64)[:, None] * 499 + torch.arange(k, device="cuda") * 262144) % classes
    top = torch.tensor([3.0, 2.0, 1.0, 0.0], device="cuda").expand(n, k).contiguous()
    got = call(z, index.to(torch.int32).contiguous(), top, None, 1.0, 1.0)
    p = torch.softmax(top[0].double(), 0)
    loss = float((p * torch.log(p)).sum()) + torch.log(torch.tensor(float(classes), dtype=torch.float64)).item()
    assert ((got["rows"].double() - loss).abs() <= TOL * 2 * loss).all()
    ref = (1.0 / classes - p) / n
    assert ((got["dz"].gather(1, index).double() - ref).abs() <= (2.0 ** -8 + TOL) * ref.abs()).all()
    assert (got["dz"] > 0).sum() == n * (classes - k)


def test_replayed_and_on_another_stream():
    n, classes, k = 70, 3001, 20
    z, index, top, lab = inputs(n, classes, k, "bf16", ragged=True, padded=True)
    ws = torch.empty(B().op_distill_workspace(n, classes, k, B().BF16), dtype=torch.uint8, device="cuda")
    rows, loss, dz = torch.empty(n, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(z)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        B().op_distill(z, index, top, lab, rows, loss, dz, 2.0, 0.5, ws, ignore=-9)
    for seed in (2, 3, 4):
        for a, b in zip((z, index, top, lab), inputs(n, classes, k, "bf16", seed=seed, ragged=True, padded=True)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = call(z, index, top, lab, 2.0, 0.5, ignore=-9)
        assert torch.equal(got["dz"], dz) and torch.equal(got["rows"], rows) and torch.equal(got["loss"], loss)


@pytest.mark.parametrize("classes,k", [(50, 3), (3000, 80), (300001, 5)])
def test_a_row_of_z_that_is_no_distribution_has_no_loss_even_without_a_list(classes, k):
    z, index, top, _ = inputs(4, classes, k, "f32")
    labels = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    z[1], index[1], index[2] = -torch.inf, -1, -1
    for alpha in (1.0, 0.5):
        out = call(z, index, top, labels, 2.0, alpha)
        assert out["rows"][1].isnan() and out["dz"][1].isnan().all() and out["loss"].isnan().all()
        assert out["rows"][[0, 2, 3]].isfinite().all() and out["dz"][[0, 2, 3]].isfinite().all()
        assert alpha < 1 or (out["rows"][2] == 0 and not out["dz"][2].any())


@pytest.mark.parametrize("temperature", [1e-18, 1e18])
def test_the_smallest_and_the_largest_temperature(temperature):
    z, index, top, _ = inputs(5, 200, 7, "f32", labels=False)
    out = call(z, index, top, None, temperature, 1.0)
    assert out["dz"].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(1, 16389, 3), (3, 33591, 19), (32, 20003, 70), (33, 20003, 70), (2, 131073, 1024), (32, 270000, 5)])
def test_few_long_rows(n, classes, k, dtype):
    for labels, alpha in ((False, 1.0), (True, 0.3)):
        x = inputs(n, classes, k, dtype, labels=labels, ragged=n > 1)
        out = call(*x, 2.0, alpha)
        agree(out, reference(*x, 2.0, alpha), dtype)
        assert torch.equal(call(*x, 2.0, alpha, inplace=True)["dz"], out["dz"])
