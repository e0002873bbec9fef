"""Sizes that pass 32 bits are refused by the binding, not taken modulo 2^32."""
import pytest
import torch

from paper_1901_06773_amd import binding as B

MANY = (1 << 32) + 5


def test_workspaces():
    assert B.op_glu_workspace(5, 16, 16, True) > 0 and B.op_distill_workspace(5, 1, 1) > 0 and B.op_linear_ce_workspace(5, 16, 10, True) > 0 and B.op_gn_workspace(5, 4, 8, 2) > 0
    assert B.op_top_logits_workspace(5, 200000, 3) > 0
    for size in (B.op_glu_workspace(MANY, 16, 16, True), B.op_glu_workspace(5, MANY, 16, False), B.op_distill_workspace(MANY, 1, 1), B.op_distill_workspace(5, 10, MANY),
                 B.op_top_logits_workspace(MANY, 200000, 3), B.op_top_logits_workspace(5, 200000 + (1 << 32), 3), B.op_linear_ce_workspace(MANY, 16, 10, True),
                 B.op_linear_ce_workspace(5, 16, 10 + (1 << 32), True), B.op_gn_workspace(MANY, 4, 8, 2), B.op_gn_workspace(5, 4 + (1 << 32), 8, 2)):
        assert size == 0


@pytest.mark.gpu
def test_calls():
    half, dev = torch.bfloat16, "cuda"
    x, h = torch.empty(MANY, 1, dtype=half, device=dev), torch.full((MANY, 1), 7.0, dtype=half, device=dev)
    w, ws = torch.zeros(2, 1, dtype=half, device=dev), torch.empty(1 << 20, dtype=torch.uint8, device=dev)
    dw = torch.empty(2, 1, device=dev)
    index, top = torch.zeros(MANY, 1, dtype=torch.int32, device=dev), torch.zeros(MANY, 1, device=dev)
    loss = torch.full((1,), 7.0, device=dev)
    for call in (lambda: B.op_glu_fwd(x, w, None, h, None, 0, ws), lambda: B.op_glu_bwd(x, w, None, None, h, None, dw, None, 0, ws), lambda: B.op_top_logits(x, index, top, ws),
                 lambda: B.op_distill(x, index, top, None, None, loss, None, 1.0, 1.0, ws), lambda: B.op_linear_ce(x, w, None, index.view(-1), None, loss, None, None, None, ws),
                 lambda: B.op_gn_fwd(x, dw[0], dw[0], None, h, top, top, 1, 0, 1e-5, ws),
                 lambda: B.op_gn_bwd(x, x, None, None, dw[0], dw[0], top, top, h, dw[0], dw[1], None, 1, 0, ws)):
        with pytest.raises(B.AccError):
            call()
    torch.cuda.synchronize()
    assert (h[:10] == 7).all() and loss == 7 and not index[:10].any() and not top[:10].any()
