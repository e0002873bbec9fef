"""The k largest logits of each row against a stable sort: whole numbers and copies of values, so that everything has to be equal."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def B():
    from paper_1901_06773_amd import binding
    return binding


def logits(n, classes, dtype, seed=1, spread=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (spread * torch.randn(n, classes, generator=g, device="cuda")).to(DT[dtype])


def call(z, k):
    n, classes = z.shape
    size = B().op_top_logits_workspace(n, classes, k, B()._dtype_of(z))
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None
    index, top = torch.full((n, k), -7, dtype=torch.int32, device="cuda"), torch.full((n, k), float("nan"), device="cuda")
    B().op_top_logits(z, index, top, ws)
    return index, top


def check(z, k):
    index, top = call(z, k)
    # a stable order of whole numbers: both zeros alike, what is no number above all
    v = z.float() + 0.0
    bits = v.view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    order = torch.where(v != v, 1 << 40, order)
    want = torch.sort(order, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(index.long(), want)
    values = v.gather(1, want)
    assert torch.equal(torch.nan_to_num(top, nan=1e38), torch.nan_to_num(values, nan=1e38))


# one class, every entry, lists longer than a wave or than the threads of a row, widths that begin rows anywhere, each size of workgroup, rows in segments
SIZES = [(1, 1, 1), (3, 2, 1), (5, 2, 2), (64, 1000, 16), (9, 63, 63), (4, 257, 65), (300, 10, 3), (7, 1021, 5), (33, 2039, 200), (3, 2048, 1024), (2, 1024, 1024),
         (5, 4099, 7), (40, 8191, 300), (6, 16385, 64), (11, 30011, 511), (3, 50001, 100), (2, 65409, 1), (2, 65536, 600), (3, 131008, 64), (2, 131009, 64),
         (2, 131072, 256), (5, 1306, 118), (9, 183, 33), (9, 183, 150), (4, 2500, 900), (3, 4500, 1024), (3, 8200, 800), (3, 8192, 1024), (2, 4097, 1024),
         (3, 300007, 33), (1, 1 << 20, 1024), (2, (1 << 20) - 3, 5)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", SIZES)
def test_against_a_stable_sort(n, classes, k, dtype):
    check(logits(n, classes, dtype), k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(3, 1000, 16), (2, 5000, 300), (2, 20001, 64), (2, 70001, 1024), (2, 200003, 40)])
def test_many_equal_values(n, classes, k, dtype):
    check(torch.zeros(n, classes, device="cuda", dtype=DT[dtype]), k)                         # nothing but ties
    check((logits(n, classes, dtype) * 0.5).round(), k)                                       # a handful of values, both zeros among them
    check(-(logits(n, classes, dtype).abs().round()), k)                                      # no positive one
    z = logits(n, classes, dtype)
    z[:, ::2] = 3.5                                                                           # a plateau with values above and below it
    check(z, k)
    z = torch.full_like(z, -2.25)
    z[:, -3:] = 1.0                                                                           # few above a plateau, at the end of the row
    check(z, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(4, 77, 20), (4, 3001, 64), (4, 40001, 100), (4, 150001, 100)])
def test_values_that_are_not_finite(n, classes, k, dtype):
    z = logits(n, classes, dtype)
    z[0, 5::3] = -float("inf")                          # classes that are ruled out
    z[1, :] = -float("inf")
    z[1, classes // 2] = 0.0
    z[2, classes - 2] = float("nan")
    z[2, 1] = float("nan")
    z[2, 7] = float("inf")
    z[3, :] = float("nan")
    check(z[:n], k)


def test_offsets_beyond_32_bits():
    n, classes, k = 2100, 1 << 20, 8                    # 2.2e9 values
    z = torch.zeros(n, classes, device="cuda", dtype=torch.bfloat16)
    z[:, ::4] = -1.0
    at = (torch.arange(n, device="cuda") * 499 + 3) % classes
    z[torch.arange(n, device="cuda"), at] = 2.0
    index, top = call(z, k)
    assert torch.equal(index[:, 0].long(), at) and (top[:, 0] == 2).all() and (top[:, 1:] == 0).all()
    first = [j for j in range(20) if j % 4][:k - 1]
    rows = at > 20
    assert torch.equal(index[rows][:, 1:].long(), torch.tensor(first, device="cuda").expand(int(rows.sum()), -1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(5, 1003, 7), (3, 200003, 33)])
def test_nothing_is_written_behind_the_results(n, classes, k, dtype):
    z = logits(n, classes, dtype)
    size = B().op_top_logits_workspace(n, classes, k, B()._dtype_of(z))
    index, top = torch.full((n * k + 4096,), 77, dtype=torch.int32, device="cuda"), torch.full((n * k + 4096,), 77.0, device="cuda")
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    B().op_top_logits(z, index[:n * k].view(n, k), top[:n * k].view(n, k), ws[:size] if size else None)
    assert all((t[-4096:] == 77).all() for t in (index, top, ws))
    a, b = call(z, k)
    assert torch.equal(index[:n * k].view(n, k), a) and torch.equal(top[:n * k].view(n, k), b)


def test_replayed_and_on_another_stream():
    z, k = logits(50, 20001, "bf16"), 40
    other = torch.cuda.Stream()
    index, top = torch.empty(50, k, dtype=torch.int32, device="cuda"), torch.empty(50, k, device="cuda")
    other.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        B().op_top_logits(z, index, top, None)
    for seed in (2, 3, 4):
        z.copy_(logits(50, 20001, "bf16", seed))
        graph.replay()
        torch.cuda.synchronize()
        a, b = call(z, k)
        assert torch.equal(index, a) and torch.equal(top, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(3, 20000, 769), (2, 33001, 1000), (3, 60000, 1024)])
def test_long_lists_of_long_rows(n, classes, k, dtype):
    z = logits(n, classes, dtype)
    check(z, k)
    check(z.round(), k)
    z[0, 3:classes - k // 2] = -float("inf")            # fewer finite values than entries
    check(z, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(40, 100, 60), (40, 200, 40), (40, 259, 125), (3000, 259, 125), (3000, 1000, 50), (3, 1000, 200), (5, 2000, 200), (7, 511, 190)])
def test_rows_bounded_by_groups_of_a_thread(n, classes, k, dtype):
    z = logits(n, classes, dtype)
    check(z, k)
    check((2 * z).round(), k)
    z[0] = -float("inf")
    z[1, 1:] = -float("inf")
    z[2, ::2] = float("nan")
    check(z, k)
