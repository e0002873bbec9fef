"""Linear cross-entropy without logits against its formulas in 64 bits.

Tolerances, as norms over a tensor.  A logit is the sum of d products of fp32 (or exact bf16) values: its error against the norm of what is summed
stays under 2^-20 up to d = 4096 (d^(1/2) roundings of 2^-24 at random add to 2^-18 of one product, 1/d^(1/2) of the sum's terms' norm), and the
loss, a probability and a gradient move by as much, times the spread of the logits: 2e-5 in all.  With bf16 operands dx is made of values of
dz rounded to bf16 and is rounded to bf16 itself (2^-8 each at most), dw of dz as the sum of two bf16 values (2^-16)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = 2e-5


def B():
    from paper_1901_06773_amd import binding
    return binding


def randn(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def inputs(n, d, classes, dtype, seed=1, spread=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    w = spread / d ** 0.5 * torch.randn(classes, d, generator=g, device="cuda")
    labels = torch.randint(classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn(n, d, generator=g, device="cuda") + w[labels.long()]
    return x.to(DT[dtype]), w.to(DT[dtype]), 0.3 * torch.randn(classes, generator=g, device="cuda"), labels


def call(x, w, bias, labels, ignore=None, want=("rows", "loss", "dx", "dw", "db"), ws=None):
    n, d = x.shape
    classes = w.shape[0]
    nan = float("nan")
    out = dict(rows=torch.full((n,), nan, device="cuda"), loss=torch.full((1,), nan, device="cuda"), dx=torch.full_like(x, nan),
               dw=torch.full((classes, d), nan, device="cuda"), db=torch.full((classes,), nan, device="cuda"))
    out = {k: v if k in want else None for k, v in out.items()}
    grads = any(k in want for k in ("dx", "dw", "db"))
    if ws is None:
        ws = torch.empty(B().op_linear_ce_workspace(n, d, classes, grads, B()._dtype_of(x)), dtype=torch.uint8, device="cuda")
        ws.fill_(255)                           # NaN wherever something is read that was not written
    B().op_linear_ce(x, w, bias, labels, out["rows"], out["loss"], out["dx"], out["dw"], out["db"], ws, ignore)
    return out


def reference(x, w, bias, labels, ignore=None):
    x, w = x.double(), w.double()
    n, classes = x.shape[0], w.shape[0]
    z = x @ w.T + (bias.double() if bias is not None else 0.0)
    counts = labels != ignore if ignore is not None else torch.ones(n, dtype=torch.bool, device="cuda")
    at = labels.long().clamp(0, classes - 1)
    rows = torch.where(counts, torch.logsumexp(z, 1) - z[torch.arange(n, device="cuda"), at], 0.0)
    share = counts.double() / max(1, int(counts.sum()))
    dz = torch.softmax(z, 1)
    dz[torch.arange(n, device="cuda"), at] -= 1.0
    dz = torch.where(counts[:, None], dz, 0.0) * share[:, None]
    return dict(rows=rows, loss=(rows * share).sum().view(1), dx=dz @ w, dw=dz.T @ x, db=dz.sum(0))


def agree(got, ref, dtype):
    for k, v in got.items():
        if v is None:
            continue
        tol = TOL + (2.0 ** -7 if k == "dx" and dtype == "bf16" else 2.0 ** -16 if k == "dw" and dtype == "bf16" else 0.0)
        r = ref[k]
        floor = 1e-9                            # one class: every gradient is nothing but rounding
        assert torch.isfinite(v).all(), k
        assert (v.double() - r).norm() <= tol * r.norm() + floor * v.numel() ** 0.5, (k, float((v.double() - r).norm() / r.norm()))


def sizes():
    return [(1, 1, 1), (1, 8, 2), (2, 3, 5), (1, 512, 1000), (41, 2048, 1000), (64, 64, 64), (65, 72, 257), (3, 16, 5000), (130, 96, 513), (255, 256, 256),
            (257, 264, 1030), (200, 130, 77), (31, 1160, 4097), (1000, 40, 10), (512, 512, 512), (33, 33, 9000), (300, 1024, 3), (5, 4096, 333), (700, 136, 8200)]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", sizes())
def test_against_the_formulas(n, d, classes, dtype, bias):
    x, w, b, labels = inputs(n, d, classes, dtype)
    b = b if bias else None
    agree(call(x, w, b, labels), reference(x, w, b, labels), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", [(8000, 64, 20000), (4100, 24, 33333), (16384, 16, 9001)])
def test_several_pieces(n, d, classes, dtype):
    x, w, b, labels = inputs(n, d, classes, dtype)
    agree(call(x, w, b, labels), reference(x, w, b, labels), dtype)


# widths of one to three values, odd ones, few rows with a long sum that is cut, more rows than a launch of whole rows takes, an odd last piece
ODD = [(1, 1, 8193), (17, 2, 20000), (700, 3, 8195), (66, 57, 9001), (42, 2050, 8301), (129, 1027, 131), (20000, 9, 40), (16385, 3, 4), (8000, 61, 20001),
       (64, 4096, 8300), (2000, 17, 3), (33, 700, 16999)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", ODD)
def test_odd_widths(n, d, classes, dtype):
    x, w, b, labels = inputs(n, d, classes, dtype)
    labels[::5] = -7
    got, ref = call(x, w, b, labels, ignore=-7), reference(x, w, b, labels, ignore=-7)
    agree(got, ref, dtype)
    for k in ("rows", "dw"):
        assert torch.equal(call(x, w, b, labels, ignore=-7, want=(k,))[k], got[k]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", [(65, 57, 9001), (42, 2050, 8301), (129, 1027, 131), (7, 3, 5), (8000, 61, 20001)])
def test_nothing_is_written_behind_the_results(n, d, classes, dtype):
    x, w, b, labels = inputs(n, d, classes, dtype)
    behind = 4096

    def buffer(count, dt=torch.float32):
        return torch.full((count + behind,), 77.0, device="cuda", dtype=dt)
    size = B().op_linear_ce_workspace(n, d, classes, True, B()._dtype_of(x))
    bufs = dict(rows=buffer(n), loss=buffer(1), dx=buffer(n * d, x.dtype), dw=buffer(classes * d), db=buffer(classes),
                ws=torch.full((size + behind,), 77, device="cuda", dtype=torch.uint8))
    B().op_linear_ce(x, w, b, labels, bufs["rows"][:n], bufs["loss"][:1], bufs["dx"][:n * d].view(n, d), bufs["dw"][:classes * d].view(classes, d),
                     bufs["db"][:classes], bufs["ws"][:size])
    assert all((v[-behind:] == 77).all() for v in bufs.values())
    assert all(torch.isfinite(v).all() for k, v in bufs.items() if k != "ws")


@pytest.mark.parametrize("dtype,d", [("f32", 1031), ("bf16", 2072)])
def test_offsets_beyond_32_bits(dtype, d):
    n, classes = 24, 1100003                    # 4.5 GB of weights, and of their gradient in fp32
    x, w, b, labels = inputs(n, d, classes, dtype)
    labels[0], labels[1] = classes - 1, 0
    got = call(x, w, b, labels)
    x64, z = x.double(), torch.empty(n, classes, dtype=torch.float64, device="cuda")
    step = 100000
    for v in range(0, classes, step):
        z[:, v:v + step] = x64 @ w[v:v + step].double().T + b[v:v + step].double()
    at = (torch.arange(n, device="cuda"), labels.long())
    rows = torch.logsumexp(z, 1) - z[at]
    dz = torch.softmax(z, 1)
    dz[at] -= 1.0
    dz /= n
    dx = torch.zeros(n, d, dtype=torch.float64, device="cuda")
    for v in range(0, classes, step):
        dx += dz[:, v:v + step] @ w[v:v + step].double()
    agree({k: got[k] for k in ("rows", "loss", "dx", "db")}, dict(rows=rows, loss=rows.mean().view(1), dx=dx, db=dz.sum(0)), dtype)
    for v in (0, 400000, 1000000, classes - 1000):
        part = slice(v, v + 1000)
        agree(dict(dw=got["dw"][part]), dict(dw=dz[:, part].T @ x64), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", [(1, 64, 100), (90, 72, 300), (300, 256, 2000)])
def test_rows_that_do_not_count(n, d, classes, dtype):
    x, w, b, labels = inputs(n, d, classes, dtype)
    labels[n // 2:] = -7
    got, ref = call(x, w, b, labels, ignore=-7), reference(x, w, b, labels, ignore=-7)
    agree(got, ref, dtype)
    assert (got["rows"][n // 2:] == 0).all() and (got["dx"][n // 2:] == 0).all()
    # a class may be the one that does not count
    labels[:] = 3
    labels[0] = 4
    agree(call(x, w, b, labels, ignore=3), reference(x, w, b, labels, ignore=3), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_row_counts(dtype):
    x, w, b, labels = inputs(70, 128, 300, dtype)
    labels[:] = -1
    got = call(x, w, b, labels, ignore=-1)
    assert all((v == 0).all() for v in got.values())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", [(5, 16, 40), (90, 256, 700)])
def test_a_label_that_does_not_exist(n, d, classes, dtype):
    x, w, b, labels = inputs(n, d, classes, dtype)
    labels[1], labels[3] = classes, -1
    got = call(x, w, b, labels)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[1] = bad[3] = True
    assert torch.equal(torch.isnan(got["rows"]), bad) and torch.isnan(got["loss"]).all()
    p = torch.softmax(x.double() @ w.double().T + b.double(), 1)
    ref = (p[bad] / n) @ w.double()
    assert (got["dx"][bad].double() - ref).norm() <= (TOL + (2.0 ** -7 if dtype == "bf16" else 0)) * ref.norm()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", [(6, 32, 50), (100, 256, 1200)])
def test_classes_ruled_out_by_the_bias(n, d, classes, dtype):
    x, w, b, labels = inputs(n, d, classes, dtype)
    out = torch.arange(classes, device="cuda") % 3 == 1
    b[out] = float("-inf")
    labels = (labels // 3 * 3).int()            # never one of those
    got, ref = call(x, w, b, labels), reference(x, w, b, labels)
    agree(got, ref, dtype)
    assert (got["dw"][out] == 0).all() and (got["db"][out] == 0).all()
    b[out] = torch.finfo(torch.float32).min
    agree(call(x, w, b, labels), ref, dtype)
    # the label itself ruled out: an infinite loss, and a gradient all the same
    b[out] = float("-inf")
    labels[2] = 1
    got = call(x, w, b, labels)
    assert torch.isinf(got["rows"][2]) and got["rows"][2] > 0 and torch.isinf(got["loss"]).all() and torch.isfinite(got["dx"]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [-200.0, 200.0])
def test_large_logits(dtype, shift):
    x, w, b, labels = inputs(60, 128, 900, dtype, spread=30.0)
    b = b + shift
    z = x.double() @ w.double().T + b.double()
    got, ref = call(x, w, b, labels), reference(x, w, b, labels)
    # logits of up to 400, each off by 2^-24 of that (and of the terms it is summed from): so are rows; gradients by that, relative
    off = 16 * 2.0 ** -24 * float(z.abs().max())
    assert ((got["rows"].double() - ref["rows"]).abs() <= off).all()
    assert (got["db"].double() - ref["db"]).norm() <= 4 * off * ref["db"].norm() + 1e-9


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", [(9, 64, 100), (300, 256, 1500), (4100, 24, 33333)])
def test_each_result_alone(n, d, classes, dtype):
    x, w, b, labels = inputs(n, d, classes, dtype)
    whole = call(x, w, b, labels)
    for k in whole:
        alone = call(x, w, b, labels, want=(k,))
        assert torch.equal(alone[k], whole[k]), k
    again = call(x, w, b, labels)
    assert all(torch.equal(again[k], whole[k]) for k in whole)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_differences(dtype):
    """Gradients against central differences of the loss in 64 bits."""
    x, w, b, labels = inputs(7, 24, 19, dtype)
    got = call(x, w, b, labels)
    at = [x.double(), w.double(), b.double()]

    def loss(xv, wv, bv):
        z = xv @ wv.T + bv
        return float((torch.logsumexp(z, 1) - z.gather(1, labels.long()[:, None])[:, 0]).mean())
    for k, name in enumerate(("dx", "dw", "db")):
        g = got[name].double().view(-1)
        for i in range(0, g.numel(), max(1, g.numel() // 20)):
            hi, lo = [t.clone() for t in at], [t.clone() for t in at]
            hi[k].view(-1)[i] += 1e-5
            lo[k].view(-1)[i] -= 1e-5
            # (a dx of bf16: 2^-7 of the terms it is summed from, which its column's size bounds)
            tol = 2e-5 + (2.0 ** -7 * float(g.abs().max()) if name == "dx" and dtype == "bf16" else 0.0)
            assert abs(float(g[i]) - (loss(*hi) - loss(*lo)) / 2e-5) <= tol


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,classes", [(41, 256, 1000), (600, 512, 3000)])
def test_captured_replayed_and_on_another_stream(n, d, classes, dtype):
    x, w, b, labels = inputs(n, d, classes, dtype)
    ws = torch.empty(B().op_linear_ce_workspace(n, d, classes, True, B()._dtype_of(x)), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(x, w, b, labels, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(x, w, b, labels, ws=ws)
    for k in range(4):
        nx, nw, nb, nl = inputs(n, d, classes, dtype, seed=50 + k)
        for old, new in ((x, nx), (w, nw), (b, nb), (labels, nl)):
            old.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        got = {m: v.clone() for m, v in out.items()}
        eager = call(x, w, b, labels)
        torch.cuda.synchronize()
        assert all(torch.equal(got[m], eager[m]) for m in got)


def test_tensors_that_do_not_fit_are_refused():
    x, w, b, labels = inputs(8, 32, 20, "f32")
    good = dict(x=x, w=w, bias=b, labels=labels, rows=torch.empty(8, device="cuda"), loss=torch.empty(1, device="cuda"), dx=torch.empty_like(x),
                dw=torch.empty_like(w), db=torch.empty_like(b), ws=torch.empty(B().op_linear_ce_workspace(8, 32, 20, True, B().F32), dtype=torch.uint8, device="cuda"))
    B().op_linear_ce(*good.values())
    for bad in (dict(x=x.bfloat16()), dict(w=w.bfloat16()), dict(w=w.T), dict(labels=labels.long()), dict(labels=labels.cpu()), dict(bias=b.bfloat16()),
                dict(dw=torch.empty_like(w).bfloat16()), dict(db=torch.empty(19, device="cuda")), dict(rows=torch.empty(9, device="cuda")),
                dict(ws=torch.empty(64, dtype=torch.uint8, device="cuda")), dict(rows=None, loss=None, dx=None, dw=None, db=None)):
        with pytest.raises(B().AccError):
            B().op_linear_ce(*{**good, **bad}.values())
