"""co3_f8_weight_gradient without gradients of weights: only the sums of dy are formed."""
import pytest
import torch

import paper_2204_08211_b200 as co3
from f8_reference import TYPES, padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("clients,rows,outs,pad", [(1, 3000, 136, 0), (2, 1501, 1001, 3), (40, 300, 264, 0)])
def test_no_operands_are_written(clients, rows, outs, pad, type_):
    """The bias' bits are those of a call with weights, and of the workspace only parts of sums are touched: at most one for each 64 rows,
    4 bytes a column, where the operands would take 128 or more."""
    ins, stride = 130, outs * 130 + outs
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(clients * rows, ins, generator=gen, device="cuda")
    _, dy = padded(torch.randn(clients * rows, outs, generator=gen, device="cuda"), type_, pad, 0)
    x8 = torch.empty(co3.co3_f8_bytes(clients * rows, ins), dtype=torch.uint8, device="cuda")
    assert co3.co3_f8_pack(x, x8) == co3.OK
    ws = torch.empty(co3.co3_f8_weight_gradient_workspace_bytes(rows, outs, ins, clients), dtype=torch.uint8, device="cuda")
    both = torch.zeros(clients * stride, device="cuda")
    assert co3.co3_f8_weight_gradient(dy, x8, ins, both, both[outs * ins:], clients, stride, ws) == co3.OK
    db = torch.zeros(clients * stride, device="cuda")
    ws.fill_(0x5A)
    assert co3.co3_f8_weight_gradient(dy, x8, ins, None, db[outs * ins:], clients, stride, ws) == co3.OK
    torch.cuda.synchronize()
    by_client = lambda t: t.view(clients, stride)
    assert torch.equal(by_client(db)[:, outs * ins:], by_client(both)[:, outs * ins:])
    assert (by_client(db)[:, :outs * ins] == 0).all()
    assert (ws != 0x5A).sum() <= clients * -(-rows // 64) * outs * 4
