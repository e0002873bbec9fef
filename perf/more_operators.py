"""What the speed of the gated linear layer, of a teacher's top logits and of the distillation from them is measured on, beside
their plain forms in elementary torch operations.

A case is one pass through one operator: h = act(gate) * value of the two projections of a gated layer (forward, or its
gradients from kept or from recomputed projections), the largest logits of each row with their classes, or the distillation
loss of a student's logits from such lists with its gradient.  Sizes are those of the maps and the head of the ResNets at
224 x 224, of heads with many more classes, and single rows; drawn ones are anything of that range, ragged ones included."""
import torch

own = False                    # True: run() calls the library; False: it computes the plain form

DEV = "cuda:0"
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_ACT = {"none": 0, "relu": 1, "silu": 2}
_MOST_GLU = 12544 * 1024 * 4096
_MOST_LOGITS = 4096 * 65536


# ---------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one image's features through a gated layer, answering: latency
        dict(name="glu_fwd_bf16_1x512x2048", op="glu_fwd", dtype="bf16", rows=1, d=512, f=2048, act="silu", bias=True, keep=False),
        # 14x14 maps of 64 images, four times as wide inside, training: the projections are kept
        dict(name="glu_fwd_bf16_12544x1024x4096_kept", op="glu_fwd", dtype="bf16", rows=12544, d=1024, f=4096, act="silu", bias=False, keep=True),
        # 7x7 maps of the minibatch of the fp32 benchmark, a width that fills no tile
        dict(name="glu_fwd_f32_2009x2048x1365", op="glu_fwd", dtype="f32", rows=2009, d=2048, f=1365, act="relu", bias=True, keep=False),
        # gradients of the large layer, from its kept projections
        dict(name="glu_bwd_bf16_12544x1024x4096_kept", op="glu_bwd", dtype="bf16", rows=12544, d=1024, f=4096, act="silu", bias=False, keep=True),
        # gradients under a small memory budget: projections worked out again, rows and widths that fill nothing
        dict(name="glu_bwd_bf16_777x1160x1003", op="glu_bwd", dtype="bf16", rows=777, d=1160, f=1003, act="silu", bias=True, keep=False),
        # fp32 gradients at a minibatch of four 7x7 maps
        dict(name="glu_bwd_f32_196x512x1024", op="glu_bwd", dtype="f32", rows=196, d=512, f=1024, act="relu", bias=True, keep=False),
        # a teacher's answers to a minibatch, 1000 classes
        dict(name="top_f32_64x1000_k16", op="top", dtype="f32", n=64, classes=1000, k=16),
        # many classes
        dict(name="top_bf16_4096x65536_k64", op="top", dtype="bf16", n=4096, classes=65536, k=64),
        # rows, classes and lists that fill nothing
        dict(name="top_bf16_777x50001_k100", op="top", dtype="bf16", n=777, classes=50001, k=100),
        # head of the fp32 benchmark, labels beside the teacher
        dict(name="distill_f32_41x1000_k16", op="distill", dtype="f32", n=41, classes=1000, k=16, labels=True, padded=0.0, ragged=False, temperature=4.0, alpha=0.9),
        # many classes, the teacher alone
        dict(name="distill_bf16_4096x65536_k64", op="distill", dtype="bf16", n=4096, classes=65536, k=64, labels=False, padded=0.0, ragged=False, temperature=2.0, alpha=1.0),
        # lists of different lengths, a fifth of the rows padding
        dict(name="distill_bf16_777x50001_k100_padded", op="distill", dtype="bf16", n=777, classes=50001, k=100, labels=True, padded=0.2, ragged=True, temperature=1.0, alpha=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["glu_fwd", "glu_bwd", "top", "distill"])
    if op in ("glu_fwd", "glu_bwd"):
        while True:
            rows, d, f = _log(rng, 1, 65536), _log(rng, 16, 4096), _log(rng, 16, 8192)
            if rng.random() < 0.7:                       # widths usually come in 8s
                d, f = max(16, d // 8 * 8), max(16, f // 8 * 8)
            if rows * d * f <= _MOST_GLU and rows * (d + f) <= 12544 * 5120:
                break
        return dict(op=op, dtype=rng.choice(["f32", "bf16", "bf16"]), rows=rows, d=d, f=f, act=rng.choice(["silu", "silu", "relu", "none"]),
                    bias=rng.random() < 0.5, keep=rng.random() < 0.5)
    while True:
        n, classes, k = _log(rng, 1, 8192), _log(rng, 2, 131072), _log(rng, 1, 256)
        if n * classes <= _MOST_LOGITS and k <= classes:
            break
    case = dict(op=op, dtype=rng.choice(["f32", "bf16"]), n=n, classes=classes, k=k)
    if op == "distill":
        labels = rng.random() < 0.5
        case.update(labels=labels, padded=rng.choice([0.0, 0.0, 0.3]), ragged=rng.random() < 0.5, temperature=rng.choice([1.0, 2.0, 4.0]),
                    alpha=rng.choice([0.3, 0.5, 0.9]) if labels else 1.0)
    return case


# ---------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    make = {"glu_fwd": _prepare_glu, "glu_bwd": _prepare_glu, "top": _prepare_top, "distill": _prepare_distill}[case["op"]]
    s = make(case, gen)
    s["case"] = case
    return s


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _prepare_glu(case, gen):
    rows, d, f, dt = case["rows"], case["d"], case["f"], _DT[case["dtype"]]
    # normalised features of channels with different spreads; projections of about unit spread
    x = (_randn(gen, rows, d) * (0.5 + torch.rand(d, generator=gen, device=DEV))).to(dt)
    w = (_randn(gen, 2 * f, d) * d ** -0.5).to(dt)       # rows of the gate, then those of the value
    s = dict(x=x, w=w, bias=0.1 * _randn(gen, 2 * f) if case["bias"] else None, ab=None)
    if case["op"] == "glu_bwd":
        s["dh"] = _randn(gen, rows, f).to(dt)
        if case["keep"]:                                 # what the forward pass left behind
            s["ab"] = _plain_projections(s).to(dt)
    if own:
        from paper_1901_06773_amd import binding as B
        s["B"] = B
        kind = B.F32 if dt == torch.float32 else B.BF16
        s["ws"] = torch.empty(max(16, B.op_glu_workspace(rows, d, f, case["op"] == "glu_bwd", kind)), dtype=torch.uint8, device=DEV)
        if case["op"] == "glu_fwd":
            s["out"] = [torch.empty(rows, f, dtype=dt, device=DEV), torch.empty(rows, 2 * f, dtype=dt, device=DEV) if case["keep"] else None]
        else:
            s["out"] = [torch.empty_like(x), torch.empty(2 * f, d, device=DEV), torch.empty(2 * f, device=DEV) if case["bias"] else None]
    return s


def _logits(gen, n, classes):
    """Logits of a trained network: a broad floor and a few classes that stand out."""
    z = 2 * _randn(gen, n, classes)
    for _ in range(3):
        at = torch.randint(classes, (n, 1), generator=gen, device=DEV)
        z.scatter_add_(1, at, 4 + 4 * torch.rand(n, 1, generator=gen, device=DEV))
    return z


def _prepare_top(case, gen):
    n, classes, k, dt = case["n"], case["classes"], case["k"], _DT[case["dtype"]]
    s = dict(z=_logits(gen, n, classes).to(dt))
    if own:
        from paper_1901_06773_amd import binding as B
        s["B"] = B
        s["ws"] = torch.empty(max(16, B.op_top_logits_workspace(n, classes, k, B.F32 if dt == torch.float32 else B.BF16)), dtype=torch.uint8, device=DEV)
        s["out"] = [torch.empty(n, k, dtype=torch.int32, device=DEV), torch.empty(n, k, device=DEV)]
    return s


def _prepare_distill(case, gen):
    n, classes, k, dt = case["n"], case["classes"], case["k"], _DT[case["dtype"]]
    teacher = _logits(gen, n, classes)
    top, index = torch.topk(teacher, k, dim=1)
    # a student on its way: the teacher's logits, smaller, and its own mistakes
    z = (0.7 * teacher + _randn(gen, n, classes)).to(dt)
    del teacher
    index = index.to(torch.int32)
    if case["ragged"]:                                   # lists that end where the teacher is sure enough
        length = torch.randint(1, k + 1, (n, 1), generator=gen, device=DEV)
        index = torch.where(torch.arange(k, device=DEV) < length, index, -1)
    labels = torch.randint(classes, (n,), generator=gen, device=DEV, dtype=torch.int32) if case["labels"] else None
    if case["padded"] > 0:                               # padding at the end of a batch
        first = n - int(n * case["padded"])
        index[first:] = -1
        if labels is not None:
            labels[first:] = -1
    s = dict(z=z, index=index.contiguous(), top=top.contiguous(), labels=labels)
    if own:
        from paper_1901_06773_amd import binding as B
        s["B"] = B
        s["ws"] = torch.empty(max(16, B.op_distill_workspace(n, classes, k, B.F32 if dt == torch.float32 else B.BF16)), dtype=torch.uint8, device=DEV)
        s["out"] = [torch.empty(n, device=DEV), torch.empty(1, device=DEV), torch.empty_like(z)]
    return s


# ---------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if case["op"] == "glu_fwd":
        if own:
            h, ab = s["out"]
            s["B"].op_glu_fwd(s["x"], s["w"], s["bias"], h, ab, _ACT[case["act"]], s["ws"])
        else:
            h, ab = _plain_glu_fwd(s, case["act"], case["keep"])
        return dict(h=h, ab=ab)
    if case["op"] == "glu_bwd":
        if own:
            dx, dw, db = s["out"]
            s["B"].op_glu_bwd(s["x"], s["w"], s["bias"], s["ab"], s["dh"], dx, dw, db, _ACT[case["act"]], s["ws"])
        else:
            dx, dw, db = _plain_glu_bwd(s, case["act"])
        return dict(dx=dx, dw=dw, db=db)
    if case["op"] == "top":
        if own:
            index, top = s["out"]
            s["B"].op_top_logits(s["z"], index, top, s["ws"])
        else:
            index, top = _plain_top(s["z"], case["k"])
        return dict(index=index, top=top)
    if own:
        rows, loss, dz = s["out"]
        s["B"].op_distill(s["z"], s["index"], s["top"], s["labels"], rows, loss, dz, case["temperature"], case["alpha"], s["ws"], ignore=-1)
    else:
        rows, loss, dz = _plain_distill(s, case["temperature"], case["alpha"])
    return dict(rows=rows, loss=loss, dz=dz)


# ---------------------------------------------------------------------------------- the plain forms
def _plain_projections(s):
    ab = s["x"].float() @ s["w"].float().T
    return ab if s["bias"] is None else ab + s["bias"]


def _plain_glu_fwd(s, act, keep):
    ab = _plain_projections(s)
    a, b = ab.chunk(2, dim=1)
    if act == "relu":
        a = torch.where(a > 0, a, 0.0)
    elif act == "silu":
        a = a / (1 + torch.exp(-a))
    return (a * b).to(s["x"].dtype), ab.to(s["x"].dtype) if keep else None


def _plain_glu_bwd(s, act):
    ab = _plain_projections(s) if s["ab"] is None else s["ab"].float()
    a, b = ab.chunk(2, dim=1)
    if act == "relu":
        value, slope = torch.where(a > 0, a, 0.0), (a > 0).float()
    elif act == "silu":
        sig = 1 / (1 + torch.exp(-a))
        value, slope = a * sig, sig * (1 + a * (1 - sig))
    else:
        value, slope = a, torch.ones_like(a)
    dh = s["dh"].float()
    dab = torch.cat([dh * b * slope, dh * value], 1)
    dx = (dab @ s["w"].float()).to(s["x"].dtype)
    return dx, dab.T @ s["x"].float(), dab.sum(0) if s["bias"] is not None else None


def _plain_top(z, k):
    # a stable order leaves equal logits by their class (0.0: both zeros are equal)
    top, index = torch.sort(z.float() + 0.0, dim=1, descending=True, stable=True)
    return index[:, :k].to(torch.int32).contiguous(), top[:, :k].contiguous()


def _plain_distill(s, temperature, alpha):
    n, k = s["index"].shape
    there = s["index"] >= 0
    at = s["index"].clamp(min=0).long()
    has = there[:, :1].float()
    # the teacher, over the classes of its list
    t = torch.where(there, s["top"] / temperature, -torch.inf)
    t = t - torch.where(there[:, :1], t.max(1, keepdim=True).values, 0.0)
    e = torch.exp(t)
    total = torch.where(there[:, :1], e.sum(1, keepdim=True), 1.0)
    p = e / total
    log_p = torch.where(there, t - torch.log(total), 0.0)
    # the student, over all classes
    z = s["z"].float()
    z = z - z.max(1, keepdim=True).values
    y = torch.exp(z / temperature)
    y_sum = y.sum(1, keepdim=True)
    log_q = z.gather(1, at) / temperature - torch.log(y_sum)
    soft = temperature * temperature * (p * (log_p - log_q)).sum(1)
    dz = (alpha * temperature) * (y / y_sum * has)
    dz.scatter_add_(1, at, (-alpha * temperature) * p)
    counts = there[:, 0] if s["labels"] is None else s["labels"] >= 0
    rows = alpha * soft
    if s["labels"] is not None:
        label, every = s["labels"].clamp(min=0).long(), torch.arange(n, device=z.device)
        y = torch.exp(z)
        y_sum = y.sum(1, keepdim=True)
        rows = rows + (1 - alpha) * (torch.log(y_sum.view(n)) - z[every, label])
        dz = dz + (1 - alpha) * (y / y_sum)
        dz[every, label] -= 1 - alpha
    rows = torch.where(counts, rows, 0.0)
    each = counts.float() / counts.sum().clamp(min=1)
    return rows, (rows * each).sum().view(1), (dz * each.view(n, 1)).to(s["z"].dtype)


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("glu_fwd", "glu_bwd"):
        rows, d, f = case["rows"], case["d"], case["f"]
        if case["op"] == "glu_fwd":
            return dict(bytes=es * (rows * d + 2 * f * d + rows * f * (1 + 2 * case["keep"])) + 8 * f * case["bias"], flops=4 * rows * d * f)
        # x, w, dh and the projections (or the bias they are worked out again with) in; dx, dw and db out
        moved = es * (2 * rows * d + 2 * f * d + rows * f * (1 + 2 * case["keep"])) + 8 * f * d + 8 * f * case["bias"] * (1 + (not case["keep"]))
        return dict(bytes=moved, flops=(8 if case["keep"] else 12) * rows * d * f)
    n, classes, k = case["n"], case["classes"], case["k"]
    if case["op"] == "top":
        return dict(bytes=es * n * classes + 8 * n * k, flops=n * classes)
    return dict(bytes=2 * es * n * classes + 8 * n * k + 4 * n * (1 + case["labels"]) + 4, flops=(5 + 4 * case["labels"]) * n * classes)


# ---------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "top":
        return _exact_top(s["z"], case["k"])
    if case["op"] == "distill":
        return _exact_distill(s, case)
    f = case["f"]
    x, w = s["x"].double().requires_grad_(), s["w"].double().requires_grad_()
    bias = (s["bias"].double() if case["bias"] else torch.zeros(2 * f, dtype=torch.float64, device=DEV)).requires_grad_()
    gate, value = torch.addmm(bias[:f], x, w[:f].t()), torch.addmm(bias[f:], x, w[f:].t())
    act = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v)}[case["act"]]
    if case["op"] == "glu_fwd":
        with torch.no_grad():
            return dict(h=act(gate) * value, ab=torch.cat([gate, value], 1) if case["keep"] else None)
    if case["keep"]:
        # gradients at the kept projections: of the layer behind them, then through the products
        a = s["ab"][:, :f].double().requires_grad_()
        b = s["ab"][:, f:].double().requires_grad_()
        (act(a) * b).backward(s["dh"].double())
        torch.autograd.backward([gate, value], [a.grad, b.grad])
    else:
        (act(gate) * value).backward(s["dh"].double())
    return dict(dx=x.grad, dw=w.grad, db=bias.grad if case["bias"] else None)


def _exact_top(z, k):
    # whole keys in the order of the logits, the lower class first among equals: no two are alike
    classes = z.shape[1]
    bits = (z.float() + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    key = order * classes + (classes - 1 - torch.arange(classes, device=z.device))
    index = classes - 1 - torch.topk(key, k, dim=1).values.remainder(classes)
    return dict(index=index.to(torch.int32), top=z.gather(1, index).double())


def _exact_distill(s, case):
    z = s["z"].double().requires_grad_()
    n, classes = z.shape
    temperature, alpha = case["temperature"], case["alpha"]
    q = torch.log_softmax(z / temperature, 1)
    there = s["index"] >= 0
    listed_rows = torch.nonzero(there[:, 0]).view(-1)
    rows = torch.zeros(n, dtype=torch.float64, device=DEV)
    if len(listed_rows):
        p = torch.softmax(torch.where(there, s["top"].double() / temperature, -torch.inf)[listed_rows], 1)
        log_p = torch.where(p > 0, torch.log(p.clamp(min=1e-300)), 0.0)
        log_q = torch.take_along_dim(q[listed_rows], s["index"][listed_rows].clamp(min=0).long(), 1)
        rows = rows.index_add(0, listed_rows, alpha * temperature ** 2 * (p * (log_p - log_q)).sum(1))
    if case["labels"]:
        kept = torch.nonzero(s["labels"] >= 0).view(-1)
        hard = torch.zeros(n, dtype=torch.float64, device=DEV)
        hard = hard.index_add(0, kept, -torch.log_softmax(z[kept], 1).gather(1, s["labels"][kept].long().unsqueeze(1)).squeeze(1))
        rows = rows + (1 - alpha) * hard
    else:
        kept = listed_rows
    loss = rows[kept].sum() / max(1, len(kept)) + 0.0 * z.sum()
    loss.backward()
    return dict(rows=rows.detach(), loss=loss.detach().view(1), dz=z.grad)
