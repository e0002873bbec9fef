"""The gated layer's backward pass writes no more of [da | db] than what is asked for is multiplied from: in bf16 three values of it for dw of fewer than 10240
rows, two for dw of more and for dx, none for dbias; in fp32 the one for dx and dw, none for dbias.  What is written is seen in a workspace full of one byte."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def B():
    from paper_1901_06773_amd import binding
    return binding


def written(x, w, bias, ab, dh, want):
    """Bytes of the workspace that are others than before, and the results."""
    rows, d, f = x.shape[0], x.shape[1], w.shape[0] // 2
    ws = torch.full((B().op_glu_workspace(rows, d, f, True, B()._dtype_of(x)),), 0xEE, dtype=torch.uint8, device="cuda")
    out = dict(dx=torch.empty_like(x), dw=torch.empty(2 * f, d, device="cuda"), db=torch.empty(2 * f, device="cuda"))
    out = {k: v if k in want else None for k, v in out.items()}
    B().op_glu_bwd(x, w, bias, ab, dh, out["dx"], out["dw"], out["db"], 2, ws)
    return int((ws != 0xEE).sum()), out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,f", [(200, 64, 40), (64, 4096, 96), (131, 40, 57), (3000, 256, 512), (5000, 64, 64), (9000, 520, 264), (10240, 48, 72), (12000, 512, 1024)])
def test_nothing_that_is_not_asked_for(rows, d, f, dtype):
    g = torch.Generator(device="cuda").manual_seed(5)

    def r(*s):
        return torch.randn(*s, generator=g, device="cuda")
    x, w, bias, dh, ab = (v.to(DT[dtype]) if i != 2 else v for i, v in enumerate((r(rows, d), r(2 * f, d) / d ** 0.5, r(2 * f), r(rows, f), r(rows, 2 * f))))
    one = rows * 2 * f * (4 if dtype == "f32" else 2)      # a value of dz; some bytes are what they were
    for kept in (None, ab):
        every, out = written(x, w, bias, kept, dh, ("dx", "dw", "db"))
        if dtype == "bf16" and rows < 10240:
            dx, alone = written(x, w, bias, kept, dh, ("dx",))
            assert every - dx >= 0.95 * one
            assert torch.equal(alone["dx"], out["dx"])
        db, alone = written(x, w, bias, kept, dh, ("db",))
        assert every - db >= 0.95 * one * (1 if dtype == "f32" else 3 if rows < 10240 else 2)
        assert torch.equal(alone["db"], out["db"])
        dw, alone = written(x, w, bias, kept, dh, ("dw",))
        assert torch.equal(alone["dw"], out["dw"])
