"""co3_f8_pack, co3_f8_unpack and the activation on 8-bit blocks against the definition in 64 bits.

What is packed is compared exactly: the format says which value each entry has.  y8 alone (the blocks of act(x)) may have the
neighbouring value where act(x) lies next to a border, since act(x) is formed in fp32: it must be the packed value of
something within the error of act(x).

Tolerances of act, relative to the result, u = 2^-24.  fp32: erfcf is good to 4 u, expf to 4 u, and three roundings follow: 8 u; erfc's
argument z = x / sqrt(2) has two roundings, 2 u of z, to which erfc answers with at most 2 z^2 + 1 = x^2 + 1 times as much.
16-bit results: the fit and its evaluation 5e-6 < 2^-17; the exponent x^2 / 2 has three roundings, 3 u x^2 / 2 of the result, and SILU's
exponent x log2(e) two, 2 u |x|.  An exponential below 2^-126 may count as zero: (1 + |x|) 2^-126.  Of the slope, a sum of two
terms, the same relative to the terms' size.  The result's own rounding is added, and the smallest steps of fp16 and fp32.
"""
import math

import pytest
import torch

import paper_2204_08211_b200 as co3
from f8_reference import TYPES, UNIT, blocks, outside_untouched, padded, values

pytestmark = pytest.mark.gpu

ACTS = [co3.ACT_NONE, co3.ACT_RELU, co3.ACT_GELU, co3.ACT_SILU]
U = 2.0 ** -24
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}
KINDS = [co3.F8_ROWS, co3.F8_SQUARE]


def inputs(rows, cols, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(rows, cols, generator=gen) * torch.exp(torch.randn(cols, generator=gen)) * torch.exp(torch.randn(rows, 1, generator=gen)) * scale


def room(rows, cols, kind=co3.F8_ROWS, fill=0xCD):
    return torch.full((co3.co3_f8_bytes(rows, cols, kind) + 512,), fill, dtype=torch.uint8, device="cuda")


def act64(act, x):
    """act(x), its derivative, and the size of the derivative's terms."""
    if act == co3.ACT_RELU:
        return x.clamp(min=0), (x > 0).double(), torch.ones_like(x)
    if act == co3.ACT_GELU:
        below, term = 0.5 * torch.special.erfc(-x / math.sqrt(2)), x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        return x * below, below + term, below + term.abs()
    if act == co3.ACT_SILU:
        p = torch.sigmoid(x)
        return x * p, p * (1 + x * (1 - p)), p * (1 + (x * (1 - p)).abs())
    return x, torch.ones_like(x), torch.ones_like(x)


def slack(act, type_, x):
    """Relative error of act(x) before it is rounded."""
    if act < co3.ACT_GELU:
        return torch.zeros_like(x)
    if type_ == "f32":
        return 8 * U + (2 * U * (x * x + 1) if act == co3.ACT_GELU else 0 * x)
    return 2.0 ** -17 + U * (1.5 * x * x if act == co3.ACT_GELU else 2 * x.abs())


def lost(act, x):
    return 0 * x if act < co3.ACT_GELU else (1 + x.abs()) * 2.0 ** -126


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (2, 7), (5, 129), (16, 512), (17, 640), (127, 255), (128, 128), (129, 1032), (300, 130), (40, 5000)])
def test_values(rows, cols, kind, type_):
    """There and back, dense rows and padded ones that start anywhere; nothing is written beside them."""
    for pad, shift in ((0, 0), (3, 1), (8, 8)):
        _, x = padded(inputs(rows, cols, rows * 1000 + cols), type_, pad, shift)
        f8 = room(rows, cols, kind)
        assert co3.co3_f8_pack(x, f8, kind) == co3.OK
        want = values(x.cpu(), kind == co3.F8_SQUARE)
        for out in ("f32", "bf16"):
            ybuf, y = padded(torch.zeros(rows, cols), out, pad, (shift * 5) % 8, 9.0)
            assert co3.co3_f8_unpack(f8, y, kind) == co3.OK
            torch.cuda.synchronize()
            assert torch.equal(y.double().cpu(), want)
            assert outside_untouched(ybuf, y, 9.0)
        assert (f8[co3.co3_f8_bytes(rows, cols, kind):] == 0xCD).all()


def test_many_rows():
    """The larger unit of rows a warp, and its ragged end."""
    x = inputs(2003, 3000, 5).cuda().bfloat16()
    for kind in KINDS:
        f8, y = room(2003, 3000, kind), torch.empty_like(x)
        assert co3.co3_f8_pack(x, f8, kind) == co3.OK and co3.co3_f8_unpack(f8, y, kind) == co3.OK
        torch.cuda.synchronize()
        assert torch.equal(y.double().cpu(), values(x.cpu(), kind == co3.F8_SQUARE))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("pad", [0, 1])
def test_borders_ties_and_extremes(kind, pad):
    """Every code and every midpoint, in blocks whose maximum lies on and next to the scale's borders; fp32's largest and smallest
    values; blocks of zeros; infinities and NaN, which do not move their block's scale."""
    codes = torch.arange(128, dtype=torch.uint8).view(torch.float8_e4m3fn).float()[:127]
    line = torch.cat([codes, (codes[1:] + codes[:-1]) / 2, -codes])
    up = lambda v: torch.nextafter(torch.tensor(v), torch.tensor(math.inf)).item()
    rows = []
    for most in (448.0, up(448.0), 447.0, 256.0, 1.0, up(1.75), 3.0e38, 3.4028234663852886e38, 1.75 * 2.0 ** 127, up(1.75 * 2.0 ** 127), 2.0 ** -126, 448 * 2.0 ** -126, 2.0 ** -149):
        row = torch.zeros(384)
        row[:380] = line[:380] * min(1.0, most / 448.0 if most < 448 else 1.0)
        row[127] = row[255] = row[383] = most
        rows.append(row)
    rows.append(torch.zeros(384))
    for bad in (math.inf, -math.inf, math.nan):
        row = line[:380].clone()
        row = torch.cat([row, torch.zeros(4)])
        row[3], row[200] = bad, bad
        rows.append(row)
    rows.append(torch.full((384,), math.nan))
    if kind == co3.F8_SQUARE:  # a block of 128 rows for each
        x = torch.cat([r.expand(128, -1) for r in rows])[:-5]
    else:
        x = torch.stack(rows)
    _, v = padded(x, "f32", pad, pad)
    f8, y = room(*x.shape, kind), torch.empty(x.shape, device="cuda")
    assert co3.co3_f8_pack(v, f8, kind) == co3.OK and co3.co3_f8_unpack(f8, y, kind) == co3.OK
    torch.cuda.synchronize()
    want, got = values(x, kind == co3.F8_SQUARE), y.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    assert torch.isfinite(got[:6]).all()


@pytest.mark.parametrize("type_", ["f16", "bf16"])
def test_extremes_of_16_bits(type_):
    t = TYPES[type_]
    x = torch.zeros(4, 256, dtype=t)
    x[0, 0], x[0, 1], x[0, 2] = torch.finfo(t).max, -torch.finfo(t).max, 1.0
    x[1, 7], x[1, 8] = torch.finfo(t).tiny, torch.finfo(t).smallest_normal / 8
    x[2, 0], x[2, 255], x[2, 5] = math.inf, math.nan, 3.0
    x[3] = 5.0
    for pad in (0, 1):
        _, v = padded(x, type_, pad, 0)
        f8, y = room(4, 256), torch.empty(4, 256, device="cuda")
        assert co3.co3_f8_pack(v, f8) == co3.OK and co3.co3_f8_unpack(f8, y) == co3.OK
        torch.cuda.synchronize()
        want, got = values(x), y.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def check_y8(f8, y64, err):
    """Each block of y8 is the packed form of something within err of y64."""
    rows, cols = y64.shape
    got = torch.empty(rows, cols, device="cuda")
    assert co3.co3_f8_unpack(f8, got) == co3.OK
    torch.cuda.synchronize()
    got = got.double().cpu()
    exps, _ = blocks(y64.numpy(), False)
    step = 2.0 ** torch.from_numpy(exps).double()
    # half a step of the value's binade (2^-4 of it at most) or of the sub-normal step (2^-10 of the scale), the scale's own step up
    # where the maximum lies next to its border
    most = (y64.abs() + err) / 16 + step * 2 * 2.0 ** -10 + err
    assert ((got - y64).abs() <= most).all()


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 127, 1), (33, 512, 0), (20, 1000, 0), (150, 1030, 2)])
def test_activation(rows, cols, pad, act, type_):
    """All outputs together, each alone, and in place; the backward pass from what was kept, in place too."""
    x = inputs(rows, cols, rows + cols + act, 1.5)
    dy = inputs(rows, cols, rows + cols + act + 1, 0.1)
    _, xv = padded(x, type_, pad, pad)
    x64 = xv.double().cpu()
    y64, _, _ = act64(act, x64)
    err = slack(act, type_, x64) * y64.abs() + lost(act, x64)
    ybuf, y = padded(torch.zeros(rows, cols), type_, pad, 0, 9.0)
    x8, y8 = room(rows, cols), room(rows, cols)
    assert co3.co3_f8_activation(xv, act, y, y8, x8) == co3.OK
    torch.cuda.synchronize()
    assert ((y.double().cpu() - y64).abs() <= err + (0.0 if act < 2 else UNIT[type_] * y64.abs() + TINY[type_])).all()
    assert outside_untouched(ybuf, y, 9.0)
    check_y8(y8, y64, err)
    kept = torch.empty(rows, cols, device="cuda")
    assert co3.co3_f8_unpack(x8, kept) == co3.OK
    torch.cuda.synchronize()
    assert torch.equal(kept.double().cpu(), values(xv.cpu()))
    for outs in ((True, False, False), (False, True, False), (False, False, True)):
        z, z8, k8 = (torch.empty_like(y) if outs[0] else None), (room(rows, cols) if outs[1] else None), (room(rows, cols) if outs[2] else None)
        assert co3.co3_f8_activation(xv, act, z, z8, k8) == co3.OK
        torch.cuda.synchronize()
        if z is not None:
            assert torch.equal(z, y)
        for a, b in ((z8, y8), (k8, x8)):
            if a is not None:
                u, v = torch.empty(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
                assert co3.co3_f8_unpack(a, u) == co3.OK and co3.co3_f8_unpack(b, v) == co3.OK
                assert torch.equal(u, v)
    _, dv = padded(dy, type_, pad, 0)
    dbuf, dx = padded(torch.zeros(rows, cols), type_, pad, pad, 9.0)
    assert co3.co3_f8_activation_backward(dv, x8, act, dx) == co3.OK
    torch.cuda.synchronize()
    k64 = kept.double().cpu()
    _, slope, size = act64(act, k64)
    want = dv.double().cpu() * slope
    err = (2 * slack(act, type_, k64) * size + 2 * lost(act, k64) + U * slope.abs()) * dv.double().cpu().abs() + UNIT[type_] * want.abs() + TINY[type_]
    assert ((dx.double().cpu() - want).abs() <= err).all()
    assert outside_untouched(dbuf, dx, 9.0)
    assert co3.co3_f8_activation_backward(dv, x8, act, dv) == co3.OK            # over dy
    torch.cuda.synchronize()
    assert torch.equal(dv, dx)
    assert co3.co3_f8_activation(xv, act, xv, None, None) == co3.OK             # over x
    torch.cuda.synchronize()
    assert torch.equal(xv, y)


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("act", ACTS[1:])
def test_activation_of_extremes(act, type_):
    """Far out on both sides and at zero; infinities give the limits, NaN stays and spoils nothing else; their kept form is NaN."""
    line = torch.cat([torch.linspace(-12, 12, 97), torch.tensor([0.0, -0.0, 100.0, -100.0, 3.0e4, -3.0e4])])
    x = torch.zeros(2, 128)
    x[0, :line.numel()] = line
    x[1, :3] = torch.tensor([math.inf, -math.inf, math.nan])
    _, xv = padded(x, type_, 0, 0)
    y, x8 = torch.empty_like(xv), room(2, 128)
    assert co3.co3_f8_activation(xv, act, y, None, x8) == co3.OK
    dx = torch.ones_like(xv)
    assert co3.co3_f8_activation_backward(dx, x8, act, dx) == co3.OK
    torch.cuda.synchronize()
    x64 = xv[0].double().cpu()
    y64, _, _ = act64(act, x64)
    err = (slack(act, type_, x64) + UNIT[type_]) * y64.abs() + lost(act, x64) + TINY[type_]
    assert ((y[0].double().cpu() - y64).abs() <= err).all()
    assert y[1, 0] == math.inf and y[1, 1] == 0 and torch.isnan(y[1, 2]) and (y[1, 3:] == 0).all()
    assert torch.isnan(dx[1, :3]).all() and torch.isfinite(dx[1, 3:]).all() and torch.isfinite(dx[0]).all()


def test_gelu_and_silu_slopes_against_differences():
    """The backward pass against differences of the forward pass, both in fp32, at points that 8 bits hold exactly.  A step of 2^-7
    leaves h^2 / 6 times the third derivative (at most 2: 2^-15.6) and the forward's error twice over 2 h (2^-24 * 8 * 4 / 2^-6 = 2^-13)."""
    x = torch.linspace(-4, 3.75, 32).repeat(2, 4).cuda()
    h = 2.0 ** -7
    for act in (co3.ACT_GELU, co3.ACT_SILU):
        x8, up, down, dx = room(2, 128), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        assert co3.co3_f8_activation(x + h, act, up) == co3.OK and co3.co3_f8_activation(x - h, act, down) == co3.OK
        assert co3.co3_f8_pack(x, x8) == co3.OK
        assert co3.co3_f8_activation_backward(torch.ones_like(x), x8, act, dx) == co3.OK
        kept = torch.empty_like(x)
        assert co3.co3_f8_unpack(x8, kept) == co3.OK
        torch.cuda.synchronize()
        assert torch.equal(kept, x)
        assert ((up - down) / (2 * h) - dx).abs().max() <= 2.0 ** -12


def test_empty():
    x, f8 = torch.zeros(0, 16, device="cuda"), room(0, 16)
    assert co3.co3_f8_pack(x, f8) == co3.OK and co3.co3_f8_unpack(f8, x) == co3.OK
    assert co3.co3_f8_activation(x, co3.ACT_GELU, x, None, f8) == co3.OK and co3.co3_f8_activation_backward(x, f8, co3.ACT_GELU, x) == co3.OK
    torch.cuda.synchronize()
    assert (f8 == 0xCD).all()
