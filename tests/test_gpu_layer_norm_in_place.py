"""Layer norm in place, at a width of every kernel: the result may lie over x, dx over dy or over x.  The same sums are
formed in the same order, so that every output has to have the bits of the call with buffers of its own."""
import pytest
import torch

import paper_2204_08211_b200 as co3
from test_gpu_layer_norm import TYPES, inputs, rows_of

pytestmark = pytest.mark.gpu

# a warp a row, a block a row and two passes over a row, with rows on 16-byte boundaries and at any alignment
WIDTHS = [(64, 0), (1024, 0), (1023, 1), (4096, 0), (4095, 2), (8191, 0), (16384, 0), (16383, 1), (16400, 0), (20001, 3)]


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("cols,pad", WIDTHS)
def test_forward_over_x(cols, pad, type_):
    rows = 9
    x, _, w, b = inputs(rows, cols, cols)
    _, xv = rows_of(x, type_, pad, 0)
    _, y = rows_of(x, type_, pad, 0)
    stats = [torch.empty(rows, device="cuda") for _ in range(4)]
    assert co3.co3_layer_norm(xv, w, b, y, stats[0], stats[1]) == co3.OK
    assert co3.co3_layer_norm(xv, w, b, xv, stats[2], stats[3]) == co3.OK
    torch.cuda.synchronize()
    assert torch.equal(xv, y) and torch.equal(stats[0], stats[2]) and torch.equal(stats[1], stats[3])


@pytest.mark.parametrize("over", ["dy", "x"])
@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("cols,pad", WIDTHS)
def test_backward_over(cols, pad, type_, over):
    clients, rows = 2, 7
    total = clients * rows
    x, dy, w, b = inputs(total, cols, cols + 1)
    _, xv = rows_of(x, type_, pad, 0)
    _, dv = rows_of(dy, type_, pad, 0)
    _, dx = rows_of(dy, type_, pad, 0)
    mean, rstd = torch.empty(total, device="cuda"), torch.empty(total, device="cuda")
    assert co3.co3_layer_norm(xv, w, b, dx, mean, rstd) == co3.OK
    ws = torch.empty(co3.co3_layer_norm_workspace_bytes(rows, cols, clients), dtype=torch.uint8, device="cuda")
    grads = torch.zeros(2, clients, 2 * cols, device="cuda")

    def call(to, g):
        flat = g.view(-1)
        assert co3.co3_layer_norm_backward(dv, xv, w, mean, rstd, to, flat, flat[cols:], clients, 2 * cols, ws) == co3.OK
    call(dx, grads[0])
    target = dv if over == "dy" else xv
    call(target, grads[1])
    torch.cuda.synchronize()
    assert torch.equal(target, dx)
    assert torch.equal(grads[1], grads[0])
