"""co3_f8_weight_gradient against sums in 64 bits of dy and of what the kept inputs stand for.

Tolerance: the parts of dy and their products with x are exact.  The tensor core adds 16 products and the sum so far at a time and
cuts each addend 25 bits below the largest or lower: a step is off by at most 17 * 2^-25 < 2^-20.9 of S, the sum of the terms' sizes;
there are rows / 16 steps for each of at most three parts, of which the later ones are 2^-8 and 2^-16 of the first, and the sums taken out
are added to nearest.  So (rows / 16 + 3) * 2^-20.8 * S; the sums of dy are fp32 sums, at most rows additions deep.
"""
import pytest
import torch

import paper_2204_08211_b200 as co3
from f8_reference import TYPES, padded

pytestmark = pytest.mark.gpu


def room(rows, cols):
    return torch.full((co3.co3_f8_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")


def kept(rows, ins, seed):
    """Inputs in 8-bit blocks, and what they stand for."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, ins, generator=gen, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=gen, device="cuda"))
    x8, v = room(rows, ins), torch.empty(rows, ins, device="cuda")
    assert co3.co3_f8_pack(x, x8) == co3.OK and co3.co3_f8_unpack(x8, v) == co3.OK
    return x8, v.double()


def gradients(rows, outs, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    return torch.randn(rows, outs, generator=gen, device="cuda") * torch.exp(torch.randn(rows, 1, generator=gen, device="cuda")) * 0.1


def workspace(rows, outs, ins, clients):
    return torch.full((co3.co3_f8_weight_gradient_workspace_bytes(rows, outs, ins, clients),), 0xFF, dtype=torch.uint8, device="cuda")


def check(dy, v, grads, at_w, at_b, clients, stride, before=None):
    rows, (outs, ins) = dy.shape[0] // clients, (dy.shape[1], v.shape[1])
    for u in range(clients):
        d, x = dy[u * rows:(u + 1) * rows].double(), v[u * rows:(u + 1) * rows]
        for at, want, size, err in ((at_w, d.T @ x, d.abs().T @ x.abs(), (rows / 16 + 3) * 2.0 ** -20.8), (at_b, d.sum(0), d.abs().sum(0), (rows + 3) * 2.0 ** -24)):
            if at is None:
                continue
            where = slice(u * stride + at, u * stride + at + want.numel())
            got = grads[where].double().view(want.shape)
            if before is not None:
                old = before[where].double().view(want.shape)
                want, size = want + old, size + old.abs()
            assert ((got - want).abs() <= err * size + 2.0 ** -140).all(), (u, at)


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("clients,rows,ins,outs,pad", [
    (1, 1, 1, 1, 0), (1, 1, 128, 256, 0), (1, 64, 128, 128, 0), (1, 65, 129, 257, 0), (3, 101, 300, 200, 0), (2, 63, 100, 129, 1), (5, 64, 128, 384, 8),
    (1, 300, 1000, 520, 0), (2, 1501, 1023, 1001, 17), (100, 8, 64, 40, 0), (300, 1, 40, 8, 3), (1, 3000, 257, 40, 0), (1, 5000, 512, 512, 0), (1, 700, 2100, 2050, 0), (1, 256, 130, 70, 0), (1, 257, 130, 70, 1),
    (40, 33, 130, 100, 2), (1, 3, 2200, 2000, 0), (400, 1, 3, 2, 0)])
def test_sizes(clients, rows, ins, outs, pad, type_):
    """Dense and padded rows, one client and many, sizes around every tile; nothing is written beside the two layers."""
    total = clients * rows
    x8, v = kept(total, ins, rows + ins)
    _, dy = padded(gradients(total, outs, rows + outs), type_, pad, pad % 3)
    stride, at_w, at_b = outs * ins + outs + 9, 1, outs * ins + 4
    grads = torch.full((clients * stride + 8,), 5.0, device="cuda")
    ws, res = workspace(rows, outs, ins, clients), torch.zeros(co3.RESULT_DTYPE.itemsize, dtype=torch.uint8, device="cuda")
    assert co3.co3_f8_weight_gradient(dy, x8, ins, grads[at_w:], grads[at_b:], clients, stride, ws, res=res) == co3.OK
    torch.cuda.synchronize()
    assert co3.read_results(res, 1)["status"][0] == co3.OK
    check(dy, v, grads, at_w, at_b, clients, stride)
    touched = torch.zeros(grads.numel(), dtype=torch.bool, device="cuda")
    for u in range(clients):
        touched[u * stride + at_w:u * stride + at_w + outs * ins] = True
        touched[u * stride + at_b:u * stride + at_b + outs] = True
    assert (grads[~touched] == 5.0).all()
    again = torch.full_like(grads, 5.0)
    ws.fill_(0x7F)
    assert co3.co3_f8_weight_gradient(dy, x8, ins, again[at_w:], again[at_b:], clients, stride, ws) == co3.OK
    torch.cuda.synchronize()
    assert torch.equal(again, grads)                                             # the same call, the same bits


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("clients,rows,ins,outs", [(2, 200, 130, 70), (1, 4000, 130, 300), (30, 64, 256, 256)])
def test_accumulates_and_leaves_out(clients, rows, ins, outs, type_):
    total = clients * rows
    x8, v = kept(total, ins, 3)
    _, dy = padded(gradients(total, outs, 4), type_, 0, 0)
    stride = outs * ins + outs
    before = torch.randn(clients * stride, device="cuda")
    ws = workspace(rows, outs, ins, clients)
    call = lambda g, w, b: co3.co3_f8_weight_gradient(dy, x8, ins, g if w else None, g[outs * ins:] if b else None, clients, stride, ws, accumulate=True)
    both = before.clone()
    assert call(both, True, True) == co3.OK
    torch.cuda.synchronize()
    check(dy, v, both, 0, outs * ins, clients, stride, before)
    for w, b in ((True, False), (False, True), (False, False)):
        g = before.clone()
        assert call(g, w, b) == co3.OK
        torch.cuda.synchronize()
        rows_of = lambda t: (t.view(clients, stride)[:, :outs * ins], t.view(clients, stride)[:, outs * ins:])
        for part, wanted in zip(range(2), (w, b)):
            assert torch.equal(rows_of(g)[part], rows_of(both if wanted else before)[part])


@pytest.mark.parametrize("rows", [64, 512])
def test_every_bit_of_fp32_counts(rows):
    """dy whose parts of eight bits cancel in the sums but for the lowest."""
    ins, outs = 128, 128
    x8, v = room(rows, ins), torch.ones(rows, ins, device="cuda")
    assert co3.co3_f8_pack(v, x8) == co3.OK
    dy = torch.full((rows, outs), 1.0, device="cuda")
    dy[::2] = -(1.0 + 2.0 ** -23)
    grads = torch.zeros(outs * ins, device="cuda")
    assert co3.co3_f8_weight_gradient(dy, x8, ins, grads, None, 1, outs * ins, workspace(rows, outs, ins, 1)) == co3.OK
    torch.cuda.synchronize()
    # the tensor core adds up the lowest parts first: they are all of one sign; the others cancel exactly
    assert torch.equal(grads, torch.full_like(grads, -rows / 2 * 2.0 ** -23))


@pytest.mark.parametrize("rows", [130, 700])
@pytest.mark.parametrize("type_", list(TYPES))
def test_nonfinite(type_, rows):
    """An infinity of dy times inputs that are not zero, a NaN of dy, a NaN among the kept inputs: each where it belongs."""
    ins, outs = 200, 304
    x = torch.rand(rows, ins, device="cuda") + 0.5
    x[100, 7] = float("nan")
    x8 = room(rows, ins)
    assert co3.co3_f8_pack(x, x8) == co3.OK
    _, dy = padded(torch.rand(rows, outs), type_, 0, 0)
    dy[5, 11], dy[9, 40], dy[70, 200] = float("inf"), float("-inf"), float("nan")
    grads = torch.zeros(outs * ins + outs, device="cuda")
    assert co3.co3_f8_weight_gradient(dy, x8, ins, grads, grads[outs * ins:], 1, outs * ins + outs, workspace(rows, outs, ins, 1)) == co3.OK
    torch.cuda.synchronize()
    dw, db = grads[:outs * ins].view(outs, ins), grads[outs * ins:]
    nan = torch.zeros(outs, ins, dtype=torch.bool, device="cuda")
    nan[200], nan[:, 7] = True, True
    assert torch.equal(torch.isnan(dw), nan)
    others = torch.arange(ins, device="cuda") != 7
    assert (dw[11, others] == float("inf")).all() and (dw[40, others] == float("-inf")).all()
    assert db[11] == float("inf") and db[40] == float("-inf") and torch.isnan(db[200])
    fine = torch.ones(outs, dtype=torch.bool, device="cuda")
    fine[[11, 40, 200]] = False
    assert torch.isfinite(dw[fine][:, others]).all() and torch.isfinite(db[fine]).all()


def test_against_differences():
    """The gradient of sum(c * (x W^T)) with respect to W, c = dy, is linear in W: a difference quotient of the forward product's
    definition is exact but for rounding.  Entries of W are moved one at a time, in 64 bits."""
    rows, ins, outs = 40, 30, 20
    x8, v = kept(rows, ins, 7)
    dy = gradients(rows, outs, 8)
    grads = torch.zeros(outs * ins, device="cuda")
    assert co3.co3_f8_weight_gradient(dy, x8, ins, grads, None, 1, outs * ins, workspace(rows, outs, ins, 1)) == co3.OK
    torch.cuda.synchronize()
    f = lambda w: (dy.double() * (v @ w.T)).sum()
    w = torch.randn(outs, ins, dtype=torch.float64, device="cuda")
    for o, i in ((0, 0), (19, 29), (7, 3), (11, 28)):
        step = torch.zeros_like(w)
        step[o, i] = 0.5
        d = f(w + step) - f(w - step)
        size = (dy[:, o].double().abs() * v[:, i].abs()).sum()
        assert (grads.view(outs, ins)[o, i].double() - d).abs() <= (rows / 16 + 3) * 2.0 ** -20.8 * size + 1e-9 * f(w.abs()).abs()


def test_bias_alone():
    """Without weights: no inputs are needed; a layer without inputs has a bias all the same."""
    for rows, outs in ((40, 24), (3000, 136)):
        dy = gradients(2 * rows, outs, rows)
        for ins in (0, 16):
            grads = torch.full((2 * (outs + 3),), 7.0, device="cuda")
            assert co3.co3_f8_weight_gradient(dy, None, ins, None, grads, 2, outs + 3, workspace(rows, outs, ins, 2)) == co3.OK
            torch.cuda.synchronize()
            for u in range(2):
                d = dy[u * rows:(u + 1) * rows].double()
                got = grads[u * (outs + 3):(u + 1) * (outs + 3)]
                assert ((got[:outs].double() - d.sum(0)).abs() <= (rows + 3) * 2.0 ** -24 * d.abs().sum(0)).all() and (got[outs:] == 7.0).all()


def test_no_rows():
    grads = torch.full((2 * 40,), 7.0, device="cuda")
    dy, x8, ws = torch.zeros(0, 8, device="cuda"), room(0, 4), workspace(0, 8, 4, 2)
    assert co3.co3_f8_weight_gradient(dy, x8, 4, grads, grads[32:], 2, 40, ws, accumulate=True) == co3.OK
    torch.cuda.synchronize()
    assert (grads == 7.0).all()
    assert co3.co3_f8_weight_gradient(dy, x8, 4, grads, grads[32:], 2, 40, ws) == co3.OK
    torch.cuda.synchronize()
    assert (grads == 0.0).all()


def test_captured_on_another_stream_and_many_in_a_row():
    sizes = [(1, 64, 128, 256), (20, 30, 200, 100), (1, 4000, 300, 520)]
    cases = []
    for clients, rows, ins, outs in sizes:
        x8, v = kept(clients * rows, ins, rows)
        dy = gradients(clients * rows, outs, rows).bfloat16()
        stride = outs * ins + outs
        g = torch.zeros(clients * stride, device="cuda")
        args = (dy, x8, ins, g, g[outs * ins:], clients, stride, workspace(rows, outs, ins, clients))
        assert co3.co3_f8_weight_gradient(*args) == co3.OK
        cases.append((args, g, g.clone()))
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for k in range(60):
        for args, g, want in cases:
            g.zero_()
            assert co3.co3_f8_weight_gradient(*args) == co3.OK
            wrong += (g != want).any()
    assert wrong.item() == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for args, g, _ in cases:
            assert co3.co3_f8_weight_gradient(*args) == co3.OK
    side = torch.cuda.Stream()
    for _, g, _ in cases:
        g.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.replay()
    side.synchronize()
    for _, g, want in cases:
        assert torch.equal(g, want)


def test_binding_refusals():
    dy, x8, g = torch.zeros(6, 8, device="cuda"), room(6, 4), torch.zeros(40, device="cuda")
    ws = workspace(6, 8, 4, 1)
    for call in (lambda: co3.co3_f8_weight_gradient(dy, x8, 4, g[9:], None, 1, 32, ws), lambda: co3.co3_f8_weight_gradient(dy, x8, 4, g, g[33:], 1, 32, ws),
                 lambda: co3.co3_f8_weight_gradient(dy, x8, 4, g, None, 4, 32, ws), lambda: co3.co3_f8_weight_gradient(dy, x8, 4, g, None, 2, -32, ws),
                 lambda: co3.co3_f8_weight_gradient(dy, x8, -4, g, None, 1, 32, ws), lambda: co3.co3_f8_weight_gradient(dy, x8, 4, g.double(), None, 1, 32, ws)):
        with pytest.raises(ValueError):
            call()
    assert co3.co3_f8_weight_gradient(dy, x8[:256], 4, g, None, 1, 32, ws) == co3.ERR_CAPACITY
    assert co3.co3_f8_weight_gradient(dy, x8, 4, g, None, 1, 32, ws[:256]) == co3.ERR_CAPACITY
    torch.cuda.synchronize()
    assert (g == 0).all()
