"""co3_f8_linear, both ways, against the products of what its operands stand for in 64 bits.

Tolerance: products of two e4m3 values and scales are exact.  The tensor core adds 32 of them and the sum so far at a time and cuts
each addend 25 bits below the largest or lower, so that a step is off by at most 33 * 2^-25 < 2^-19.9 of S, the sum of the terms'
sizes; there are cols / 32 steps, and the sums taken out and the bias are added to nearest (2^-24 each).  So
(cols / 32 + 2) * 2^-19.9 * S, and half a step of y's type.
"""
import numpy as np
import pytest
import torch

import paper_2204_08211_b200 as co3
from f8_reference import TYPES, UNIT, outside_untouched, padded, values

pytestmark = pytest.mark.gpu


def room(rows, cols, kind=co3.F8_ROWS):
    """Filled with what would be NaN as a value and as a scale."""
    return torch.full((co3.co3_f8_bytes(rows, cols, kind),), 0xFF, dtype=torch.uint8, device="cuda")


def unpacked(f8, rows, cols, kind=co3.F8_ROWS):
    y = torch.empty(rows, cols, device="cuda")
    assert co3.co3_f8_unpack(f8, y, kind) == co3.OK
    return y.double()


def inputs(rows, ins, outs, transposed, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    cols = outs if transposed else ins
    x = randn(rows, cols) * torch.exp(randn(cols)) * torch.exp(randn(rows, 1))
    # blocks of the weights with very different scales
    w = randn(outs, ins) * torch.exp2(torch.randint(-9, 9, (-(-outs // 128), -(-ins // 128)), generator=gen, device="cuda").float()
                                      ).repeat_interleave(128, 0)[:outs].repeat_interleave(128, 1)[:, :ins]
    return x, w, randn(ins if transposed else outs)


def check(x8, w8, bias, y, rows, ins, outs, transposed, type_):
    cols = outs if transposed else ins
    xv, wv = unpacked(x8, rows, cols), unpacked(w8, outs, ins, co3.F8_SQUARE)
    if not transposed:
        wv = wv.T
    want, size = xv @ wv, xv.abs() @ wv.abs()
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    tiny = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}[type_]
    err = (cols / 32 + 2) * 2.0 ** -19.9 * size + UNIT[type_] * want.abs() + tiny
    assert ((y.double() - want).abs() <= err).all()


def run(rows, ins, outs, transposed, type_, pad=0, shift=0, bias=True, seed=0):
    x, w, b = inputs(rows, ins, outs, transposed, seed + rows * 7 + ins * 3 + outs)
    if type_ == "f16":
        w, x = w / 2.0 ** 12, x / 8
    cols, to = (outs, ins) if transposed else (ins, outs)
    _, xv = padded(x, type_, pad, shift)
    ybuf, y = padded(torch.zeros(rows, to), type_, pad, (3 * shift) % 8, 9.0)
    x8, w8 = room(rows, cols), room(outs, ins, co3.F8_SQUARE)
    assert co3.co3_f8_pack(w, w8, co3.F8_SQUARE) == co3.OK
    b = b if bias else None
    res = torch.zeros(co3.RESULT_DTYPE.itemsize, dtype=torch.uint8, device="cuda")
    assert co3.co3_f8_linear(xv, x8, w8, b, y, transposed, res=res) == co3.OK
    torch.cuda.synchronize()
    assert co3.read_results(res, 1)["status"][0] == co3.OK
    check(x8, w8, b, y, rows, ins, outs, transposed, type_)
    assert outside_untouched(ybuf, y, 9.0)
    z = torch.empty_like(y)                                        # from the blocks alone: the same bits
    assert co3.co3_f8_linear(None, x8, w8, b, z, transposed, cols=cols) == co3.OK
    torch.cuda.synchronize()
    assert torch.equal(z, y)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("ins,outs", [(1, 1), (127, 129), (128, 128), (129, 127), (520, 384), (1000, 1500), (4104, 300)])
@pytest.mark.parametrize("rows", [1, 2, 16, 17, 64, 65, 128, 129, 300])
def test_sizes(rows, ins, outs, transposed):
    run(rows, ins, outs, transposed, ("f32", "f16", "bf16")[(rows + ins) % 3], pad=(rows + outs) % 2, shift=rows % 3)


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,ins,outs", [(1501, 1023, 1001), (2500, 2100, 1300), (2600, 1300, 2170), (5000, 260, 2050), (2560, 2200, 4500), (40000, 100, 70)])
def test_large(rows, ins, outs, transposed, type_):
    """Tiles of every kind, their ragged ends, an odd number of them, sums that are taken out on the way."""
    run(rows, ins, outs, transposed, type_, bias=not transposed)


@pytest.mark.parametrize("rows", [1, 7, 16])
@pytest.mark.parametrize("ins,outs", [(9000, 130), (4300, 9600), (128 * 64, 9600), (40000, 130)])
def test_few_rows_of_long_sums(ins, outs, rows):
    """Sums divided among the blocks of a cluster, and ones too long for that."""
    run(rows, ins, outs, False, ("f32", "f16", "bf16")[rows % 3], pad=rows % 2)
    run(rows, outs, ins, True, ("f32", "f16", "bf16")[(rows + 1) % 3], bias=False)


def test_small_sums_next_to_large_ones():
    """One row of x against all others far smaller: rows do not see each other's scales."""
    x = torch.full((200, 256), 1e-20, device="cuda")
    x[7] = 1e20
    w = torch.ones(130, 256, device="cuda")
    x8, w8, y = room(200, 256), room(130, 256, co3.F8_SQUARE), torch.empty(200, 130, device="cuda")
    assert co3.co3_f8_pack(w, w8, co3.F8_SQUARE) == co3.OK and co3.co3_f8_linear(x, x8, w8, None, y) == co3.OK
    torch.cuda.synchronize()
    check(x8, w8, None, y, 200, 256, 130, False, "f32")
    assert (y[7] > 1e22).all() and (y[8] < 1e-17).all()


@pytest.mark.parametrize("rows", [3, 100, 2600])
def test_scales_far_apart_on_both_sides(rows):
    """Very small inputs times very large weights and the other way round: only the product has to be in range."""
    ins, outs = 300, 2300
    x, w, _ = inputs(rows, ins, outs, False, 2)
    for up in (2.0 ** 90, 2.0 ** -90):
        x8, w8, y = room(rows, ins), room(outs, ins, co3.F8_SQUARE), torch.empty(rows, outs, device="cuda")
        assert co3.co3_f8_pack(w * up, w8, co3.F8_SQUARE) == co3.OK and co3.co3_f8_linear(x / up, x8, w8, None, y) == co3.OK
        torch.cuda.synchronize()
        check(x8, w8, None, y, rows, ins, outs, False, "f32")


@pytest.mark.parametrize("rows", [5, 100, 2600])
def test_nonfinite(rows):
    """A NaN or an infinity spoils its own row of x, or its own feature, and nothing else."""
    ins, outs = 300, 2300
    x, w, _ = inputs(rows, ins, outs, False, 1)
    x[2, 5], x[4, 299] = float("nan"), float("inf")
    w[130, 7] = float("-inf")
    x8, w8, y = room(rows, ins), room(outs, ins, co3.F8_SQUARE), torch.empty(rows, outs, device="cuda")
    assert co3.co3_f8_pack(w, w8, co3.F8_SQUARE) == co3.OK and co3.co3_f8_linear(x, x8, w8, None, y) == co3.OK
    torch.cuda.synchronize()
    bad = torch.zeros(rows, outs, dtype=torch.bool, device="cuda")
    bad[2], bad[4], bad[:, 130] = True, True, True
    assert torch.equal(torch.isnan(y), bad) and torch.isfinite(y[~bad]).all()


def test_against_the_definition():
    """One small product from the definition of the format itself, without the library's unpacking."""
    x, w, b = inputs(33, 200, 150, False, 5)
    x8, w8, y = room(33, 200), room(150, 200, co3.F8_SQUARE), torch.empty(33, 150, device="cuda")
    assert co3.co3_f8_pack(w, w8, co3.F8_SQUARE) == co3.OK and co3.co3_f8_linear(x, x8, w8, b, y) == co3.OK
    torch.cuda.synchronize()
    xv, wv = values(x), values(w, True)
    want, size = xv @ wv.T + b.double().cpu(), xv.abs() @ wv.T.abs() + b.double().cpu().abs()
    assert ((y.double().cpu() - want).abs() <= (200 / 32 + 2) * 2.0 ** -19.9 * size).all()


@pytest.mark.parametrize("rows", [3, 200, 3000])
def test_captured_replayed_and_on_another_stream(rows):
    ins, outs = 500, 1700
    x, w, b = inputs(rows, ins, outs, False, 9)
    x8, w8, y = room(rows, ins), room(outs, ins, co3.F8_SQUARE), torch.empty(rows, outs, device="cuda")
    assert co3.co3_f8_pack(w, w8, co3.F8_SQUARE) == co3.OK and co3.co3_f8_linear(x, x8, w8, b, y) == co3.OK
    torch.cuda.synchronize()
    want = y.clone()
    side = torch.cuda.Stream()
    y.zero_()
    side.wait_stream(torch.cuda.current_stream())
    assert co3.co3_f8_linear(x, x8, w8, b, y, stream=side) == co3.OK
    side.synchronize()
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert co3.co3_f8_linear(x, x8, w8, b, y) == co3.OK
    for k in (1.0, 2.0):
        x.mul_(k)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y - b, y - b) and torch.isfinite(y).all()
    x2 = torch.empty_like(y)
    assert co3.co3_f8_linear(x, x8, w8, b, x2) == co3.OK
    torch.cuda.synchronize()
    assert torch.equal(x2, y)


def test_many_calls_in_a_row():
    """Three hundred calls of three sizes that follow one another without a wait: each has the bits of its first run."""
    sizes = [(1, 700, 900), (150, 400, 300), (2600, 300, 2300)]
    cases = []
    for rows, ins, outs in sizes:
        x, w, b = inputs(rows, ins, outs, False, rows)
        x8, w8, y = room(rows, ins), room(outs, ins, co3.F8_SQUARE), torch.empty(rows, outs, device="cuda")
        assert co3.co3_f8_pack(w, w8, co3.F8_SQUARE) == co3.OK and co3.co3_f8_linear(x, x8, w8, b, y) == co3.OK
        cases.append((x, x8, w8, b, y, y.clone()))
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for k in range(100):
        for x, x8, w8, b, y, want in cases:
            y.zero_()
            assert co3.co3_f8_linear(x, x8, w8, b, y) == co3.OK
            wrong += (y != want).any()
    assert wrong.item() == 0


def test_empty_and_refusals():
    y = torch.zeros(0, 8, device="cuda")
    f8 = room(8, 8, co3.F8_SQUARE)
    assert co3.co3_f8_linear(y, f8, f8, None, y) == co3.OK
    a = torch.zeros(4, 8, device="cuda")
    for call in (lambda: co3.co3_f8_linear(None, f8, f8, None, a), lambda: co3.co3_f8_linear(a[:3], f8, f8, None, a),
                 lambda: co3.co3_f8_linear(a, f8, f8, torch.zeros(7, device="cuda"), a), lambda: co3.co3_f8_linear(a, f8, f8, None, a, cols=9),
                 lambda: co3.co3_f8_linear(a, f8.float(), f8, None, a), lambda: co3.co3_f8_linear(a.double(), f8, f8, None, a)):
        with pytest.raises(ValueError):
            call()
    assert co3.co3_f8_linear(a, f8[:256], f8, None, a) == co3.ERR_CAPACITY
    assert co3.co3_f8_linear(a, f8[16:], f8, None, a) == co3.ERR_INVALID_ARG
