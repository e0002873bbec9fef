"""How the gated layer, the top logits and the distillation loss are called: tensors that the binding refuses, and several streams at once."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def B():
    from paper_1901_06773_amd import binding
    return binding


def tensors():
    dev = dict(device="cuda")
    n, d, f, classes, k = 6, 16, 8, 20, 4
    return dict(x=torch.randn(n, d, **dev), w=torch.randn(2 * f, d, **dev), bias=torch.randn(2 * f, **dev), h=torch.empty(n, f, **dev), ab=torch.empty(n, 2 * f, **dev),
                dh=torch.randn(n, f, **dev), dx=torch.empty(n, d, **dev), dw=torch.empty(2 * f, d, **dev), db=torch.empty(2 * f, **dev), z=torch.randn(n, classes, **dev),
                index=torch.zeros(n, k, dtype=torch.int32, **dev), top=torch.zeros(n, k, **dev), labels=torch.zeros(n, dtype=torch.int32, **dev),
                rows=torch.empty(n, **dev), loss=torch.empty(1, **dev), dz=torch.empty(n, classes, **dev), ws=torch.empty(1 << 20, dtype=torch.uint8, **dev))


CALLS = {
    "glu_fwd": (("x", "w", "bias", "h", "ab"), lambda b, t: b.op_glu_fwd(t["x"], t["w"], t["bias"], t["h"], t["ab"], 2, t["ws"])),
    "glu_bwd": (("x", "w", "bias", "ab", "dh", "dx", "dw", "db"),
                lambda b, t: b.op_glu_bwd(t["x"], t["w"], t["bias"], t["ab"], t["dh"], t["dx"], t["dw"], t["db"], 2, t["ws"])),
    "top": (("z", "index", "top"), lambda b, t: b.op_top_logits(t["z"], t["index"], t["top"], t["ws"])),
    "distill": (("z", "index", "top", "labels", "rows", "loss", "dz"),
                lambda b, t: b.op_distill(t["z"], t["index"], t["top"], t["labels"], t["rows"], t["loss"], t["dz"], 2.0, 0.5, t["ws"])),
}


@pytest.mark.parametrize("call,name", [(c, n) for c, (names, _) in CALLS.items() for n in names])
def test_tensors_that_do_not_fit(call, name):
    run = CALLS[call][1]
    good = tensors()
    run(B(), good)                                      # as they are they fit
    t = good[name]
    wide = torch.zeros(t.shape[0], 2 * t[0].numel() if t.dim() > 1 else 2, device="cuda", dtype=t.dtype)
    bad = [t.cpu(), t.double() if t.dtype != torch.int32 else t.long(), (wide[:, ::2] if t.dim() > 1 else wide[:, 0]) if t.numel() > 1 else torch.zeros(2, device="cuda")]
    if name not in ("x", "z", "w", "index"):            # (those say what the sizes are)
        bad.append(torch.zeros(*(s + 1 for s in t.shape), device="cuda", dtype=t.dtype))
    for v in bad:
        with pytest.raises((B().AccError, TypeError)):
            run(B(), {**good, name: v})
    with pytest.raises(B().AccError):
        run(B(), {**good, "ws": good["ws"].cpu()})
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_several_streams_at_once(dtype):
    b = B()
    n, d, f, classes, k = 700, 256, 264, 5003, 30
    kind = b.F32 if dtype == torch.float32 else b.BF16

    def job(seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        t = dict(x=torch.randn(n, d, generator=g, device="cuda").to(dtype), w=(torch.randn(2 * f, d, generator=g, device="cuda") / 16).to(dtype),
                 dh=torch.randn(n, f, generator=g, device="cuda").to(dtype), z=torch.randn(n, classes, generator=g, device="cuda").to(dtype))
        t.update(h=torch.empty(n, f, device="cuda", dtype=dtype), dx=torch.empty_like(t["x"]), dw=torch.empty(2 * f, d, device="cuda"),
                 db=torch.empty(2 * f, device="cuda"), index=torch.empty(n, k, dtype=torch.int32, device="cuda"), top=torch.empty(n, k, device="cuda"),
                 rows=torch.empty(n, device="cuda"), loss=torch.empty(1, device="cuda"), dz=torch.empty_like(t["z"]))
        size = max(b.op_glu_workspace(n, d, f, True, kind), b.op_glu_workspace(n, d, f, False, kind), b.op_distill_workspace(n, classes, k, kind))
        t["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        return t

    def run(t):
        b.op_glu_fwd(t["x"], t["w"], None, t["h"], None, 2, t["ws"])
        b.op_glu_bwd(t["x"], t["w"], None, None, t["dh"], t["dx"], t["dw"], t["db"], 2, t["ws"])
        b.op_top_logits(t["z"], t["index"], t["top"], None)
        b.op_distill(t["z"], t["index"], t["top"], None, t["rows"], t["loss"], t["dz"], 2.0, 1.0, t["ws"])
    names = ("h", "dx", "dw", "db", "index", "top", "rows", "loss", "dz")
    jobs = [job(s) for s in range(3)]
    want = []
    for t in jobs:
        run(t)
        torch.cuda.synchronize()
        want.append({a: t[a].clone() for a in names})
        for a in names:
            t[a].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(3):
        for s, t in zip(streams, jobs):
            with torch.cuda.stream(s):
                run(t)
    torch.cuda.synchronize()
    for t, w in zip(jobs, want):
        for a in names:
            assert torch.equal(t[a], w[a]), a
